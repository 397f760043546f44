// Attention of few queries over many keys: new tokens over a cache.
//
// The query heads that share a key head are rows (row r: query r / G, head r % G of the group), 8 or 16 to a tile of
// mma.sync, with the keys along M and the rows along N: S^T = K Q^T, O^T = V^T P^T.  Each warp keeps its own running
// maximum, sum and output over 16 keys at a time; a block joins its warps', and where a row tile's keys are
// split over blocks, the last of them to finish joins the blocks', in order.
//
// Bound by HBM: keys and values are read once, straight into the registers of the products.  A lane's 16 bytes of a key
// are the k-indices it feeds, in an order that the queries follow; its 16 bytes of a value are eight columns, pairs
// of keys being put together by byte permutes, and the weights turned over by movmatrix.  The next keys are loaded
// before the softmax and the next values behind the products.  (tcgen05 would need 128 rows where there are 16 at
// most, and the way through shared memory.)
//
// The work is split by what there is: every block sums up the sequences' lengths and takes an equal share of
// all units of 64 keys, so that sequences of different lengths leave no SM idle.
//
// 64 sequences of 4,096 to 8,192 keys, 16 query and 4 key heads of 128, one query each: 0.127 ms, 6.4 TB/s, 94 % of the
// copy rate; eight of up to 131,072 with three queries (16 rows, 250 registers, eight warps to an SM): 0.155 ms,
// 5.3 TB/s.  One query over 1,028 keys: 9.7 us, seven of them dependent loads and the join.  Blocks of a fixed number
// of keys with the rows along M took 0.230 and 0.485 ms and 16.6 us.
#pragma once
#include "attend_tile.cuh"

namespace gnn {

constexpr int kFewWarps = 4, kFewUnit = 16 * kFewWarps;      // keys that a block takes at a time
constexpr int kFewSeqs = 1024;       // sequences whose lengths a block sums up; with more, blocks take whole row tiles
constexpr int kFewRows = 16;         // rows of a tile, at most
constexpr int kFewPadded = 8;        // shares up to which blocks have parts of one tile only

struct FewGrid {
  int group;                         // query heads to a key head
  int row_tiles;
  float* parts;                      // [block][2]: a tile's outputs [rows][dim], maxima [rows] and sums [rows]
  int* tickets;                      // [block], zero between calls: of the tile that starts in the block and goes on
};

__device__ __forceinline__ void mma_16x8x16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1, __nv_bfloat16) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16x8x16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1, __half) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 8 x 8 words of 16 bits, lane 4 r + c holding row r's columns 2c and 2c + 1, turned over.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ uint4 load_once(const char* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t word(const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

// Keys that some query of the sequence sees: [0, first) and [lo, lo + n - first).
struct FewKeys { int first, lo, n; };
__device__ __forceinline__ FewKeys few_keys(const AttendParams& p, const Sequence& sq) {
  const Seen a = seen_keys(sq.len - sq.nq, sq.len, p.left, p.right, p.sinks);
  const Seen z = seen_keys(sq.len - 1, sq.len, p.left, p.right, p.sinks);
  FewKeys k;
  k.lo = min(a.lo, z.hi);
  k.first = min(p.sinks, k.lo);
  k.n = k.first + z.hi - k.lo;
  return k;
}
__device__ __forceinline__ int few_units(const AttendParams& p, const Sequence& sq) {
  return sq.nq == 0 ? 0 : max(1, (int)(((int64_t)few_keys(p, sq).n + kFewUnit - 1) / kFewUnit));
}

// Units before each sequence (pre[0 .. n_seqs]), the first sequences (seq_s), and a block's share of all units.  A
// block whose share is small would spend it on waiting if it had parts of two tiles: there each tile starts with a block
// of its own.  128 sequences' units fit 32 bits, as each has below 2^25 - 127; those of all need not, as sequences may
// read the same keys.
template <int NR>
__device__ __forceinline__ int64_t few_share(const AttendParams& p, int KR, int64_t* pre, uint32_t* scan_s, Sequence* seq_s) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto block_scan = [&](uint32_t x, uint32_t* sum) {   // the sum up to this thread's, and that of all
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 31) scan_s[warp] = x;
    __syncthreads();
    *sum = 0;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      if (w < warp) x += scan_s[w];
      *sum += scan_s[w];
    }
    return x;
  };
  // More parts make a tile's own time shorter and its join longer (0.7 us a unit, up to 0.35 us a part of 16 rows): no
  // more than balances the two.  (One sequence of 8,192 keys, four queries, 16 rows: 41 -> 22 us.)
  auto even = [&](int64_t sum) {
    const int64_t least = (int64_t)sqrtf(0.12f * NR * (float)sum / (float)p.n_seqs);
    return max(max((int64_t)1, least), (sum * KR + gridDim.x - 1) / gridDim.x);
  };
  int64_t share = 1, before = 0;
  for (int b0 = 0; b0 < p.n_seqs; b0 += 32 * kFewWarps) {
    const int b = b0 + threadIdx.x;
    uint32_t u = 0, sum;
    if (b < p.n_seqs) {
      bool bad;
      const Sequence sq = sequence(p, b, &bad);
      if ((bad || sq.nq > p.max_q) && blockIdx.x == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
      if (b < 32 * kFewWarps) seq_s[b] = sq;
      u = few_units(p, sq);
    }
    uint32_t upto = block_scan(u, &sum);
    if (p.n_seqs <= 32 * kFewWarps) {
      share = even(sum);
      if (share <= kFewPadded) {
        for (uint32_t s = (uint32_t)share; s <= 2 * kFewPadded; ++s) {
          uint32_t padded;
          const uint32_t x = block_scan((u + s - 1) / s * s, &padded);
          if ((int64_t)padded * KR > (int64_t)s * gridDim.x) continue;
          upto = x;
          u = (u + s - 1) / s * s;
          sum = padded;
          share = s;
          break;
        }
      }
    }
    if (b < p.n_seqs) pre[b] = before + upto - u;
    before += sum;
  }
  if (threadIdx.x == 0) pre[p.n_seqs] = before;
  __syncthreads();
  return p.n_seqs > 32 * kFewWarps ? even(before) : share;
}

// NC: 16-byte pieces of a key that a lane takes, a quarter of those of head_dim up to 32 NC.  NR: rows of a tile / 8.
template <typename T, int NC, int NR>
__global__ void __launch_bounds__(32 * kFewWarps, NR == 2 && NC > 2 ? 2 : 3)
    attend_few_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ FewGrid f) {
  constexpr int NV = (NC + 1) / 2, DS = NV * 64 + 4, ROWS = 8 * NR;   // pieces of a value to a lane; a row in shared memory
  __shared__ __align__(16) float o_s[kFewWarps][ROWS][DS];
  __shared__ float m_s[kFewWarps][ROWS], l_s[kFewWarps][ROWS], sum_s[ROWS];
  __shared__ int64_t pre[kFewSeqs + 1];
  __shared__ uint32_t scan_s[kFewWarps];
  __shared__ int last_s;
  __shared__ Sequence seq_s[32 * kFewWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int KR = p.kv_heads * f.row_tiles, G = f.group;
  const float scale = fabsf(p.scale_log2), slack = 8.f / scale;       // as in the tiled kernel
  const bool balanced = p.n_seqs <= kFewSeqs;
  pdl_wait();

  const int64_t share = balanced ? few_share<NR>(p, KR, pre, scan_s, seq_s) : 1;

  // Units [v0, v1) of the `units` of row tile kr of sequence b; u0: the tile's first unit among all.
  auto process = [&](int b, int kr, int v0, int v1, int units, int64_t u0) {
    bool bad = false;
    const Sequence sq = balanced && b < 32 * kFewWarps ? seq_s[b] : sequence(p, b, &bad);
    if (!balanced && (bad || sq.nq > p.max_q) && threadIdx.x == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
    const int rt = kr % f.row_tiles, kv = kr / f.row_tiles, row0 = rt * ROWS;
    const int rows = min(min(sq.nq, p.max_q) * G - row0, ROWS);
    if (rows <= 0) return;
    const FewKeys keys = few_keys(p, sq);
    const int pos0 = sq.len - sq.nq, pos_first = pos0 + row0 / G, pos_last = pos0 + (row0 + rows - 1) / G;
    // queries as the second operand: row g of each eight, pieces t + 4 c
    uint4 q[NR][NC];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int row = row0 + 8 * r + g;
      const bool have = 8 * r + g < rows;
      const char* src = p.q.data + (int64_t)(sq.q0 + row / G) * p.q.row_bytes + (int64_t)(kv * G + row % G) * p.q.head_bytes;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        q[r][c] = make_uint4(0, 0, 0, 0);
        if (have && 8 * (t + 4 * c) < p.dim) q[r][c] = *reinterpret_cast<const uint4*>(src + 16 * (t + 4 * c));
        if (p.scale_log2 < 0.f) {
          q[r][c].x ^= 0x80008000u; q[r][c].y ^= 0x80008000u; q[r][c].z ^= 0x80008000u; q[r][c].w ^= 0x80008000u;
        }
      }
    }
    float o[NV][4][NR][4], m[NR][2], l[NR][2];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      m[r][0] = m[r][1] = -INFINITY;
      l[r][0] = l[r][1] = 0.f;
#pragma unroll
      for (int e = 0; e < NV; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[e][i][r][x] = 0.f;
    }
    // keys below full_hi and from full_lo on, or below the sinks, are seen by every row
    const int full_hi = p.right < 0 ? INT_MAX : (int)min((int64_t)INT_MAX, (int64_t)pos_first + p.right + 1);
    const int full_lo = p.left < 0 ? INT_MIN : (int)max((int64_t)INT_MIN, (int64_t)pos_last - p.left);

#pragma unroll 1
    for (int part = 0; part < 2; ++part) {           // the sinks, the window
      const int c0 = v0 * kFewUnit, c1 = min(keys.n, v1 * kFewUnit);
      const int jb = part ? keys.lo + max(c0, keys.first) - keys.first : c0;
      const int je = part ? keys.lo + c1 - keys.first : min(c1, keys.first);
      int j = jb + 16 * warp;
      if (j >= je) continue;
      const char* kp = p.k.data + (int64_t)(sq.k0 + j + g) * p.k.row_bytes + (int64_t)kv * p.k.head_bytes + 16 * t;
      const char* vp = p.v.data + (int64_t)(sq.k0 + j + 2 * t) * p.v.row_bytes + (int64_t)kv * p.v.head_bytes + 16 * g;
      uint4 k[2][NC], v[4][NV];
      auto load_k = [&](int at) {                    // keys g and g + 8 of the 16
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < NC; ++e) {
            k[h][e] = make_uint4(0, 0, 0, 0);
            if (at + g + 8 * h < je && 8 * (t + 4 * e) < p.dim) k[h][e] = load_once(kp + 8 * h * p.k.row_bytes + 64 * e);
          }
      };
      auto load_v = [&](int at) {                    // keys 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
          for (int e = 0; e < NV; ++e) {
            const int key = (h & 1) + 8 * (h >> 1);
            v[h][e] = make_uint4(0, 0, 0, 0);
            if (at + 2 * t + key < je && 8 * (g + 8 * e) < p.dim) v[h][e] = load_once(vp + key * p.v.row_bytes + 128 * e);
          }
      };
      load_k(j);
      load_v(j);
      for (;;) {
        float s[NR][4];                              // keys g (0, 1) and g + 8 (2, 3), rows 2t and 2t + 1 of each eight
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int x = 0; x < 4; ++x) s[r][x] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const uint32_t a0[4] = {k[0][c].x, k[1][c].x, k[0][c].y, k[1][c].y};
          const uint32_t a1[4] = {k[0][c].z, k[1][c].z, k[0][c].w, k[1][c].w};
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            mma_16x8x16(s[r], a0, q[r][c].x, q[r][c].y, T());
            mma_16x8x16(s[r], a1, q[r][c].z, q[r][c].w, T());
          }
        }
        const bool more = j + kFewUnit < je;
        kp += (int64_t)kFewUnit * p.k.row_bytes;
        if (more) load_k(j + kFewUnit);
        if (j + 16 > je || j + 16 > full_hi || (j < full_lo && j + 16 > p.sinks)) {
#pragma unroll
          for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int key = j + g + 8 * (x >> 1);
              const int64_t pos = (int64_t)pos0 + (row0 + 8 * r + 2 * t + (x & 1)) / G;
              const bool see = key < je && (p.right < 0 || key <= pos + p.right) &&
                               (p.left < 0 || key >= pos - p.left || key < p.sinks);
              s[r][x] = see ? s[r][x] : -INFINITY;
            }
        }
        float high[NR][2];
        bool grow = false;
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float h = fmaxf(s[r][x], s[r][x + 2]);
            h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 4));
            h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 8));
            high[r][x] = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 16));
            grow = grow || high[r][x] > m[r][x] + slack || (m[r][x] == -INFINITY && high[r][x] > m[r][x]);
          }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const float mn = fmaxf(m[r][x], high[r][x]);
              const float shrink = m[r][x] == -INFINITY ? 0.f : exp2_approx((m[r][x] - mn) * scale);
              m[r][x] = mn;
              l[r][x] *= shrink;
#pragma unroll
              for (int e = 0; e < NV; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  o[e][i][r][x] *= shrink;
                  o[e][i][r][x + 2] *= shrink;
                }
            }
        }
        uint32_t w[NR][2];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float off = m[r][x & 1] == -INFINITY ? 0.f : -m[r][x & 1] * scale;
            s[r][x] = exp2_approx(fmaf(s[r][x], scale, off));
            l[r][x & 1] += s[r][x];
          }
          w[r][0] = transpose_8x8(pack2<T>(s[r][0], s[r][1]));
          w[r][1] = transpose_8x8(pack2<T>(s[r][2], s[r][3]));
        }
#pragma unroll
        for (int e = 0; e < NV; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) {              // columns 2i and 2i + 1 of every lane's piece
            const uint32_t v0 = word(v[0][e], i), v1 = word(v[1][e], i), v2 = word(v[2][e], i), v3 = word(v[3][e], i);
            const uint32_t a[4] = {__byte_perm(v0, v1, 0x5410), __byte_perm(v0, v1, 0x7632), __byte_perm(v2, v3, 0x5410),
                                   __byte_perm(v2, v3, 0x7632)};
#pragma unroll
            for (int r = 0; r < NR; ++r) mma_16x8x16(o[e][i][r], a, w[r][0], w[r][1], T());
          }
        vp += (int64_t)kFewUnit * p.v.row_bytes;
        if (!more) break;
        load_v(j + kFewUnit);
        j += kFewUnit;
      }
    }

    // the warps' results to shared memory: row 8 r + 2 t + x, element 8 (g + 8 e) + 2 i + y
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = 8 * r + 2 * t + x;
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[r][x] += __shfl_xor_sync(0xffffffffu, l[r][x], d);
        if (g == 0) {
          m_s[warp][row] = m[r][x];
          l_s[warp][row] = l[r][x];
        }
#pragma unroll
        for (int e = 0; e < NV; ++e) {
          float* dst = &o_s[warp][row][8 * (g + 8 * e)];
#pragma unroll
          for (int i = 0; i < 4; i += 2)
            *reinterpret_cast<float4*>(dst + 2 * i) =
                make_float4(o[e][i][r][x], o[e][i][r][x + 2], o[e][i + 1][r][x], o[e][i + 1][r][x + 2]);
        }
      }
    __syncthreads();
    const bool whole = v0 == 0 && v1 == units;
    const int64_t size = (int64_t)ROWS * (p.dim + 2);
    float* mine = f.parts + ((int64_t)blockIdx.x * 2 + ((int64_t)blockIdx.x * share >= u0 ? 0 : 1)) * size;
    auto store = [&](int r, int d, float sum, float4 val) {
      char* out = p.out.data + (int64_t)(sq.q0 + (row0 + r) / G) * p.out.row_bytes +
                  (int64_t)(kv * G + (row0 + r) % G) * p.out.head_bytes;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      if (sum == 0.f) val = make_float4(0.f, 0.f, 0.f, 0.f);
      *reinterpret_cast<uint2*>(out + 2 * d) =
          make_uint2(pack2<T>(val.x * inv, val.y * inv), pack2<T>(val.z * inv, val.w * inv));
    };
    const int quads = p.dim / 4;
    for (int x = threadIdx.x; x < rows * quads; x += 32 * kFewWarps) {
      const int r = x / quads, d = 4 * (x - r * quads);
      float top = m_s[0][r];
#pragma unroll
      for (int w = 1; w < kFewWarps; ++w) top = fmaxf(top, m_s[w][r]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
      float4 val = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) {
        const float z = exp2_approx((m_s[w][r] - ref) * scale);
        const float4 y = *reinterpret_cast<const float4*>(&o_s[w][r][d]);
        sum = fmaf(l_s[w][r], z, sum);
        val.x = fmaf(y.x, z, val.x); val.y = fmaf(y.y, z, val.y); val.z = fmaf(y.z, z, val.z); val.w = fmaf(y.w, z, val.w);
      }
      if (whole) {
        store(r, d, sum, val);
      } else {
        *reinterpret_cast<float4*>(mine + r * p.dim + d) = val;
        if (d == 0) {
          mine[ROWS * p.dim + r] = top;
          mine[ROWS * p.dim + ROWS + r] = sum;
        }
      }
    }
    if (!whole) {
      const int64_t b0 = u0 / share, b1 = (u0 + units - 1) / share;   // the blocks that have a part of the tile
      const int parts = (int)(b1 - b0) + 1;
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) last_s = atomicAdd(&f.tickets[b0], 1) == parts - 1;
      __syncthreads();
      if (!last_s) return;
      __threadfence();
      if (threadIdx.x == 0) f.tickets[b0] = 0;
      // the first block's part may be its last piece of work, the others' is their first
      const float* all = f.parts + b0 * 2 * size;
      auto at = [&](int i) { return all + (2 * (int64_t)i + (i == 0 && b0 * share < u0 ? 1 : 0)) * size; };
      float* z_s = &o_s[0][0][0];                    // [rows][parts]: what each part's sums are multiplied by
      const bool fits = rows * parts <= kFewWarps * ROWS * DS;
      if (parts <= 128 && fits) {                    // all maxima and sums at once: the loads wait for nothing
        float pm[ROWS / kFewWarps][4], pl[ROWS / kFewWarps][4];
#pragma unroll
        for (int y = 0; y < ROWS / kFewWarps; ++y)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = warp + kFewWarps * y, i = lane + 32 * k;
            const bool have = r < rows && i < parts;
            pm[y][k] = have ? __ldcg(at(i) + ROWS * p.dim + r) : -INFINITY;
            pl[y][k] = have ? __ldcg(at(i) + ROWS * p.dim + ROWS + r) : 0.f;
          }
#pragma unroll
        for (int y = 0; y < ROWS / kFewWarps; ++y) {
          const int r = warp + kFewWarps * y;
          float top = fmaxf(fmaxf(pm[y][0], pm[y][1]), fmaxf(pm[y][2], pm[y][3])), sum = 0.f;
#pragma unroll
          for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float z = exp2_approx((pm[y][k] - ref) * scale);
            sum = fmaf(pl[y][k], z, sum);
            if (r < rows && lane + 32 * k < parts) z_s[r * parts + lane + 32 * k] = z;
          }
#pragma unroll
          for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
          if (lane == 0 && r < rows) sum_s[r] = sum;
        }
      } else {
        for (int r = warp; r < rows; r += kFewWarps) {
          float top = -INFINITY, sum = 0.f;
          for (int i = lane; i < parts; i += 32) top = fmaxf(top, __ldcg(at(i) + ROWS * p.dim + r));
#pragma unroll
          for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          const float ref = top == -INFINITY ? 0.f : top;
          for (int i = lane; i < parts; i += 32) {
            const float z = exp2_approx((__ldcg(at(i) + ROWS * p.dim + r) - ref) * scale);
            sum = fmaf(__ldcg(at(i) + ROWS * p.dim + ROWS + r), z, sum);
            if (fits) z_s[r * parts + i] = z;
          }
#pragma unroll
          for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
          if (lane == 0) {
            sum_s[r] = sum;
            m_s[0][r] = ref;
          }
        }
      }
      __syncthreads();
      // four outputs to a thread's place; eight parts' are loaded together
      for (int place = threadIdx.x; place < rows * quads; place += 32 * kFewWarps) {
        const int r = place / quads;
        float4 val = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i0 = 0; i0 < parts; i0 += 8) {
          float4 x[8];
          float z[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = __ldcg(reinterpret_cast<const float4*>(at(min(i0 + k, parts - 1))) + place);
          if (fits) {
#pragma unroll
            for (int k = 0; k < 8; ++k) z[k] = i0 + k < parts ? z_s[r * parts + i0 + k] : 0.f;
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              z[k] = i0 + k < parts ? exp2_approx((__ldcg(at(i0 + k) + ROWS * p.dim + r) - m_s[0][r]) * scale) : 0.f;
          }
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (i0 + k < parts) {
              val.x = fmaf(x[k].x, z[k], val.x); val.y = fmaf(x[k].y, z[k], val.y);
              val.z = fmaf(x[k].z, z[k], val.z); val.w = fmaf(x[k].w, z[k], val.w);
            }
        }
        store(r, 4 * (place - r * quads), sum_s[r], val);
      }
    }
    // A sequence's queries see different keys, all of which a tile goes through (one of a single query too), and a weight of
    // zero times a value that is not finite is NaN: such rows are done again, key by visible key.
    if (sq.nq > 1) {
      __syncthreads();
      for (int r = warp; r < rows; r += kFewWarps) {
        const int i = (row0 + r) / G, head = kv * G + (row0 + r) % G;
        const T* out = reinterpret_cast<const T*>(p.out.data + (int64_t)(sq.q0 + i) * p.out.row_bytes +
                                                  (int64_t)head * p.out.head_bytes);
        bool odd = false;
        for (int d = lane; d < p.dim; d += 32) odd = odd || !(fabsf(to_f(out[d])) < INFINITY);
        if (!__any_sync(0xffffffffu, odd)) continue;
        const T* src = reinterpret_cast<const T*>(p.q.data + (int64_t)(sq.q0 + i) * p.q.row_bytes +
                                                  (int64_t)head * p.q.head_bytes);
        float* qs = &o_s[warp][0][0];
        __syncwarp();
        for (int d = lane; d < p.dim; d += 32) qs[d] = to_f(src[d]);
        __syncwarp();
        attend_row<T>(p, sq, i, head, qs);
        __syncwarp();
      }
    }
  };

  if (balanced) {
    const int64_t end = min(((int64_t)blockIdx.x + 1) * share, pre[p.n_seqs] * KR);
    for (int64_t u = (int64_t)blockIdx.x * share; u < end;) {
      const int64_t x = u / KR;
      int a = 0, z = p.n_seqs;                       // the last sequence that starts at or before x has units
      while (z - a > 1) {
        const int mid = (a + z) / 2;
        if (pre[mid] <= x) a = mid; else z = mid;
      }
      const int units = (int)(pre[a + 1] - pre[a]);
      const int64_t r = u - pre[a] * KR;
      const int kr = (int)(r / units), v0 = (int)(r - (int64_t)kr * units), v1 = (int)min((int64_t)units, v0 + (end - u));
      // where tiles are padded to whole shares, `units` counts the padding too
      const int real = share <= 2 * kFewPadded && p.n_seqs <= 32 * kFewWarps ? few_units(p, seq_s[a]) : units;
      if (v0 < real) process(a, kr, v0, min(v1, real), real, u - v0);
      u += v1 - v0;
      __syncthreads();
    }
  } else {
    for (int64_t tile = blockIdx.x; tile < (int64_t)p.n_seqs * KR; tile += gridDim.x) {
      const int b = (int)(tile / KR);
      bool bad;
      const int units = few_units(p, sequence(p, b, &bad));
      if (bad && threadIdx.x == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
      if (units > 0) process(b, (int)(tile - (int64_t)b * KR), 0, units, units, 0);
      __syncthreads();
    }
  }
}

}  // namespace gnn
