// Attention of new queries over keys and values in pages, of hypotheses that share their first keys.
//
// Position j of sequence b lies in row table[b][j / page] * page + j % page.  Sequences come in groups; the first
// `shared` positions of a group's sequences are the same and are read through the group's first sequence's pages.
// Query i of nq of a sequence with len positions stands at p = len - nq + i and sees the keys j <= p:
// o = sum_j softmax_j(scale q.k_j) v_j; a query that sees none gets zeros.  What a query does not see takes no part in
// its result, whatever it holds.
#pragma once
#include "rotary.cuh"

namespace gnn {

struct PagedParams {
  HeadsView q, k, v, out;
  const int *q_start, *kv_len, *table;               // [n_seqs + 1], [n_seqs], [n_seqs] rows of `width` entries
  const int *group_start, *shared_len;               // [n_groups + 1], [n_groups]
  int64_t table_stride, n_pages;
  int n_q_rows, n_seqs, n_groups, width, shift;      // pages have 2^shift rows
  int max_q, heads, kv_heads, dim;
  float scale_log2;                                  // scale * log2(e)
  uint32_t* err;
};

struct PagedSequence { int q0, nq, len, group, first, shared; };   // first: whose pages the keys below `shared` are read through

// The positions that a row of the table can hold.
__device__ __forceinline__ int paged_room(const PagedParams& p) {
  return (int)min((int64_t)p.width << p.shift, (int64_t)INT_MAX >> 1);
}
// Rows [q0, q1) of sequence b, cut to the array; *bad when they were not inside.
__device__ __forceinline__ int2 paged_queries(const PagedParams& p, int b, bool* bad) {
  const int a = p.q_start[b], z = p.q_start[b + 1];
  const int q0 = min(max(a, 0), p.n_q_rows), q1 = min(max(z, q0), p.n_q_rows);
  *bad = *bad || a != q0 || z != q1;
  return make_int2(q0, q1);
}
__device__ __forceinline__ int paged_shared(const PagedParams& p, int g, bool* bad) {
  const int n = p.shared_len[g], cut = min(max(n, 0), paged_room(p));
  *bad = *bad || n != cut;
  return cut;
}
__device__ __forceinline__ PagedSequence paged_sequence(const PagedParams& p, int b, bool* bad) {
  // The group that sequence b would be of if all were as large is looked at beside the sequence itself: one round of loads.
  PagedSequence s;
  int g = -1, g0 = 0, g1 = 0, shared = 0;
  if (p.n_groups > 0) {
    g = min((int)((float)b / (float)p.n_seqs * (float)p.n_groups), p.n_groups - 1);
    g0 = p.group_start[g];
    g1 = p.group_start[g + 1];
    shared = p.shared_len[g];
  }
  const int len = p.kv_len[b];
  const int2 q = paged_queries(p, b, bad);
  s.q0 = q.x;
  s.nq = q.y - q.x;
  s.len = min(max(len, 0), paged_room(p));
  *bad = *bad || len != s.len;
  s.first = b;
  s.shared = 0;
  if (g >= 0 && !(b >= g0 && b < g1)) {
    g = sequence_of(p.group_start, p.n_groups, p.n_seqs, b);
    if (g >= 0) {
      g0 = p.group_start[g];
      shared = p.shared_len[g];
    }
  }
  s.group = g;
  if (g >= 0) {
    s.first = max(g0, 0);
    s.shared = min(max(shared, 0), paged_room(p));
    *bad = *bad || shared != s.shared;
  }
  return s;
}

// The row of position j in the pages of sequence b, or -1 where its page is none.
__device__ __forceinline__ int64_t paged_row(const PagedParams& p, int b, int j) {
  const int page = p.table[(int64_t)b * p.table_stride + (j >> p.shift)];
  return page >= 0 && page < p.n_pages ? ((int64_t)page << p.shift) + (j & ((1 << p.shift) - 1)) : -1;
}

// One query row of one head by one warp: 32 keys at a time, a key to a lane for the scores, the head's elements
// spread over the lanes for the values.  q: the row in fp32, in shared memory.
template <typename T>
__device__ __noinline__ void paged_attend_row(const PagedParams& p, const PagedSequence& sq, int b, int i, int head, const float* q) {
  const int lane = threadIdx.x & 31, kv = head / (p.heads / p.kv_heads);
  const int n = (int)max((int64_t)0, (int64_t)sq.len - sq.nq + i + 1);
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int base = 0; base < n; base += 32) {
    const int j = base + lane;
    int64_t row = -1;
    float x = -INFINITY;
    if (j < n) {
      row = paged_row(p, j < sq.shared ? sq.first : b, j);
      if (row < 0) {
        atomicOr(p.err, DEV_ERR_INDEX_RANGE);
      } else {
        const char* k_row = p.k.data + row * p.k.row_bytes + kv * p.k.head_bytes;
        x = 0.f;
        for (int d = 0; d < p.dim; d += 8) {
          const Pack<T, 8> k = *reinterpret_cast<const Pack<T, 8>*>(k_row + d * sizeof(T));
#pragma unroll
          for (int e = 0; e < 8; ++e) x = fmaf(q[d + e], to_f(k.v[e]), x);
        }
        x *= p.scale_log2;
      }
    }
    float top = x;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn;
    const float shrink = exp2f(m - ref), w = row >= 0 ? exp2f(x - ref) : 0.f;
    m = mn;
    l = l * shrink + w;
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] *= shrink;
    for (int r = 0; r < min(32, n - base); ++r) {
      const float wr = __shfl_sync(0xffffffffu, w, r);
      const int64_t at = __shfl_sync(0xffffffffu, row, r);
      if (at < 0) continue;
      const T* v_row = reinterpret_cast<const T*>(p.v.data + at * p.v.row_bytes + kv * p.v.head_bytes);
#pragma unroll
      for (int d = 0; d < 4; ++d)
        if (lane + 32 * d < p.dim) o[d] = fmaf(wr, to_f(v_row[lane + 32 * d]), o[d]);
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
  T* out = reinterpret_cast<T*>(p.out.data + (int64_t)(sq.q0 + i) * p.out.row_bytes + head * p.out.head_bytes);
#pragma unroll
  for (int d = 0; d < 4; ++d)
    if (lane + 32 * d < p.dim) out[lane + 32 * d] = from_f<T>(l == 0.f ? 0.f : o[d] / l);
}

}  // namespace gnn
