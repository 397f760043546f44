// Attention of few queries over many keys: new tokens over a cache.
//
// The query heads that share a key head are the 16 rows of an mma.sync tile (row r: query r / G, head r % G of
// the group), and the keys that any of them sees are split over blocks and, 16 at a time, over a block's warps.
// Each warp keeps its own running maximum, sum and output; a block joins its warps', and the last block of a row
// tile to finish joins the blocks', in order.
//
// Bound by HBM: keys and values are read once, straight into the registers of the products.  A lane's 16 bytes
// of a key are the k-indices it feeds, in an order that the queries follow; its 16 bytes of a value are eight
// columns, pairs of keys being put together by byte permutes.  (tcgen05 would need 128 rows where there are
// 16 at most, and the copy through shared memory.)
#pragma once
#include "attend_tile.cuh"

namespace gnn {

constexpr int kFewWarps = 4, kFewRows = 16, kFewStep = 16 * kFewWarps;   // keys that a block takes at a time

struct FewGrid {
  int group;                         // query heads to a key head
  int max_q;                         // queries of a sequence, at most
  int row_tiles, splits;             // of 16 rows; blocks along the keys, at most
  int chunk;                         // keys of a block, at least
  float* parts;                      // [item][16][dim + 2]: outputs, maximum, sum
  int* tickets;                      // per row tile, zero between calls
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
__device__ __forceinline__ uint4 load_once(const char* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

// NC: 16-byte pieces of a key that a lane takes, a quarter of those of head_dim up to 32 NC.
template <typename T, int NC>
__global__ void __launch_bounds__(32 * kFewWarps, NC > 2 ? 3 : 4)
    attend_few_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ FewGrid f) {
  constexpr int NV = (NC + 1) / 2, DS = NV * 64 + 4;       // pieces of a value to a lane; a row in shared memory
  __shared__ float o_s[kFewWarps][kFewRows][DS];
  __shared__ float m_s[kFewWarps][kFewRows], l_s[kFewWarps][kFewRows];
  __shared__ int last_s;
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x % f.splits, tile = blockIdx.x / f.splits;   // tile: sequence, key head, row tile
  const int rt = tile % f.row_tiles, at = tile / f.row_tiles, kv = at % p.kv_heads, b = at / p.kv_heads;
  bool bad;
  const Sequence sq = sequence(p, b, &bad);
  if ((bad || sq.nq > f.max_q) && threadIdx.x == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
  const int G = f.group, rows = min(min(sq.nq, f.max_q) * G - rt * kFewRows, kFewRows);
  if (rows <= 0) return;
  const int q_first = rt * kFewRows / G, q_last = (rt * kFewRows + rows - 1) / G;
  // keys that some row sees: [0, first) and [lo, hi)
  const int pos0 = sq.len - sq.nq;
  const Seen sa = seen_keys(pos0 + q_first, sq.len, p.left, p.right, p.sinks);
  const Seen sz = seen_keys(pos0 + q_last, sq.len, p.left, p.right, p.sinks);
  const int hi = sz.hi, lo = min(sa.lo, hi), first = min(p.sinks, lo), n = first + hi - lo;
  const int per = (n + f.splits - 1) / f.splits;
  const int chunk = max(f.chunk, (per + kFewStep - 1) / kFewStep * kFewStep);
  const int parts = max(1, (n + chunk - 1) / chunk);
  if (split >= parts) return;
  const int c_end = min(n, (split + 1) * chunk);

  // queries: rows g and g + 8, the pieces 8 (t + 4 c) .. + 7 of a head
  uint32_t q[NC][2][4];
  int row_pos[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = rt * kFewRows + g + 8 * h, i = r / G, head = kv * G + r % G;
    const bool have = g + 8 * h < rows;
    row_pos[h] = have ? pos0 + i : INT_MIN;
    const char* src = p.q.data + (int64_t)(sq.q0 + i) * p.q.row_bytes + (int64_t)head * p.q.head_bytes;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (have && 8 * (t + 4 * c) < p.dim) v = *reinterpret_cast<const uint4*>(src + 16 * (t + 4 * c));
      q[c][h][0] = v.x; q[c][h][1] = v.y; q[c][h][2] = v.z; q[c][h][3] = v.w;
    }
  }
  const char* kp = p.k.data + (int64_t)sq.k0 * p.k.row_bytes + (int64_t)kv * p.k.head_bytes;
  const char* vp = p.v.data + (int64_t)sq.k0 * p.v.row_bytes + (int64_t)kv * p.v.head_bytes;
  auto key_at = [&](int c) { return c < first ? c : lo + (c - first); };
  uint4 k[2][NC], v[4][NV];
  auto load_k = [&](int c0) {                              // keys g and g + 8 of the 16
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = c0 + g + 8 * h;
      const char* src = kp + (int64_t)key_at(c) * p.k.row_bytes;
#pragma unroll
      for (int e = 0; e < NC; ++e) {
        k[h][e] = make_uint4(0, 0, 0, 0);
        if (c < c_end && 8 * (t + 4 * e) < p.dim) k[h][e] = load_once(src + 16 * (t + 4 * e));
      }
    }
  };
  auto load_v = [&](int c0) {                              // keys 2t, 2t + 1, 2t + 8, 2t + 9, pieces g + 8 e
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int c = c0 + 2 * t + (h & 1) + 8 * (h >> 1);
      const char* src = vp + (int64_t)key_at(c) * p.v.row_bytes;
#pragma unroll
      for (int e = 0; e < NV; ++e) {
        v[h][e] = make_uint4(0, 0, 0, 0);
        if (c < c_end && 8 * (g + 8 * e) < p.dim) v[h][e] = load_once(src + 16 * (g + 8 * e));
      }
    }
  };
  float o[NV][8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < NV; ++e)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[e][i][x] = 0.f;

  int c0 = split * chunk + warp * 16;
  if (c0 < c_end) {
    load_k(c0);
    load_v(c0);
  }
  for (; c0 < c_end; c0 += kFewStep) {
    float s[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int x = 0; x < 4; ++x) s[h][x] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const uint32_t a0[4] = {q[c][0][0], q[c][1][0], q[c][0][1], q[c][1][1]};
        const uint32_t a1[4] = {q[c][0][2], q[c][1][2], q[c][0][3], q[c][1][3]};
        mma_16x8x16(s[h], a0, k[h][c].x, k[h][c].y, T());
        mma_16x8x16(s[h], a1, k[h][c].z, k[h][c].w, T());
      }
    }
    if (c0 + kFewStep < c_end) load_k(c0 + kFewStep);
    // s[h][x]: row g + 8 (x / 2), key 8 h + 2 t + x % 2
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int c = c0 + 8 * h + 2 * t + (x & 1), j = key_at(c);
        const int64_t pos = row_pos[x >> 1];
        const bool see = c < c_end && row_pos[x >> 1] != INT_MIN && (p.right < 0 || j <= pos + p.right) &&
                         (p.left < 0 || j >= pos - p.left || j < p.sinks);
        s[h][x] = see ? s[h][x] * p.scale_log2 : -INFINITY;
        top[x >> 1] = fmaxf(top[x >> 1], s[h][x]);
      }
    float shrink[2], ref[2];
    bool grow = false;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
      top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
      const float mn = fmaxf(m[r], top[r]);
      grow = grow || mn > m[r];
      ref[r] = mn == -INFINITY ? 0.f : mn;
      shrink[r] = exp2_approx(m[r] - ref[r]);
      m[r] = mn;
    }
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) l[r] *= shrink[r];
#pragma unroll
      for (int e = 0; e < NV; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[e][i][x] *= shrink[x >> 1];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        s[h][x] = exp2_approx(s[h][x] - ref[x >> 1]);
        l[x >> 1] += s[h][x];
      }
    const uint32_t a[4] = {pack2<T>(s[0][0], s[0][1]), pack2<T>(s[0][2], s[0][3]), pack2<T>(s[1][0], s[1][1]),
                           pack2<T>(s[1][2], s[1][3])};
#pragma unroll
    for (int e = 0; e < NV; ++e) {
      auto word = [](const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; };
#pragma unroll
      for (int i = 0; i < 8; ++i) {                        // column i of every lane's piece
        const uint32_t pick = i & 1 ? 0x7632u : 0x5410u;
        const uint32_t b0 = __byte_perm(word(v[0][e], i / 2), word(v[1][e], i / 2), pick);
        const uint32_t b1 = __byte_perm(word(v[2][e], i / 2), word(v[3][e], i / 2), pick);
        mma_16x8x16(o[e][i], a, b0, b1, T());
      }
    }
    if (c0 + kFewStep < c_end) load_v(c0 + kFewStep);
  }

  // the warps' results to shared memory: row g + 8 r, element 8 (2 t + x + 8 e) + i
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    if (t == 0) {
      m_s[warp][g + 8 * r] = m[r];
      l_s[warp][g + 8 * r] = l[r];
    }
#pragma unroll
    for (int e = 0; e < NV; ++e)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float* dst = &o_s[warp][g + 8 * r][8 * (2 * t + x + 8 * e)];
#pragma unroll
        for (int i = 0; i < 8; i += 4)
          *reinterpret_cast<float4*>(dst + i) =
              make_float4(o[e][i][2 * r + x], o[e][i + 1][2 * r + x], o[e][i + 2][2 * r + x], o[e][i + 3][2 * r + x]);
      }
  }
  __syncthreads();
  const int width = p.dim + 2;
  float* mine = f.parts + (int64_t)blockIdx.x * kFewRows * width;
  auto store = [&](int r, int d, float sum, float val) {
    T* out = reinterpret_cast<T*>(p.out.data + (int64_t)(sq.q0 + (rt * kFewRows + r) / G) * p.out.row_bytes +
                                  (int64_t)(kv * G + (rt * kFewRows + r) % G) * p.out.head_bytes);
    out[d] = from_f<T>(sum == 0.f ? 0.f : val / sum);
  };
  for (int x = threadIdx.x; x < rows * p.dim; x += 32 * kFewWarps) {
    const int r = x / p.dim, d = x - r * p.dim;
    float top = m_s[0][r];
#pragma unroll
    for (int w = 1; w < kFewWarps; ++w) top = fmaxf(top, m_s[w][r]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, val = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float z = exp2_approx(m_s[w][r] - ref);
      sum = fmaf(l_s[w][r], z, sum);
      val = fmaf(o_s[w][r][d], z, val);
    }
    if (parts == 1) {
      store(r, d, sum, val);
    } else {
      mine[r * width + d] = val;
      if (d == 0) {
        mine[r * width + p.dim] = top;
        mine[r * width + p.dim + 1] = sum;
      }
    }
  }
  if (parts > 1) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last_s = atomicAdd(&f.tickets[tile], 1) == parts - 1;
    __syncthreads();
    if (!last_s) return;
    __threadfence();
    if (threadIdx.x == 0) f.tickets[tile] = 0;
    const float* all = f.parts + (int64_t)tile * f.splits * kFewRows * width;
    const int64_t step = (int64_t)kFewRows * width;
    for (int x = threadIdx.x; x < rows * p.dim; x += 32 * kFewWarps) {
      const int r = x / p.dim, d = x - r * p.dim;
      const float* at_r = all + r * width;
      float top = -INFINITY;
      for (int i = 0; i < parts; ++i) top = fmaxf(top, __ldcg(at_r + i * step + p.dim));
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f, val = 0.f;
      for (int i = 0; i < parts; ++i) {
        const float z = exp2_approx(__ldcg(at_r + i * step + p.dim) - ref);
        sum = fmaf(__ldcg(at_r + i * step + p.dim + 1), z, sum);
        val = fmaf(__ldcg(at_r + i * step + d), z, val);
      }
      store(r, d, sum, val);
    }
  }
  // Rows of several queries see different keys, and a weight of zero times a value that is not finite is NaN: such
  // rows are done again, key by visible key.
  if (q_last > q_first) {
    __syncthreads();
    for (int r = warp; r < rows; r += kFewWarps) {
      const int i = (rt * kFewRows + r) / G, head = kv * G + (rt * kFewRows + r) % G;
      const T* out = reinterpret_cast<const T*>(p.out.data + (int64_t)(sq.q0 + i) * p.out.row_bytes +
                                                (int64_t)head * p.out.head_bytes);
      bool odd = false;
      for (int d = lane; d < p.dim; d += 32) odd = odd || !(fabsf(to_f(out[d])) < INFINITY);
      if (!__any_sync(0xffffffffu, odd)) continue;
      const T* src = reinterpret_cast<const T*>(p.q.data + (int64_t)(sq.q0 + i) * p.q.row_bytes +
                                                (int64_t)head * p.q.head_bytes);
      float* qs = &o_s[warp][0][0];
      for (int d = lane; d < p.dim; d += 32) qs[d] = to_f(src[d]);
      __syncwarp();
      attend_row<T>(p, sq, i, head, qs);
      __syncwarp();
    }
  }
}

}  // namespace gnn
