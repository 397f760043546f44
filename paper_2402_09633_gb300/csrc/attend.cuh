// Attention with a sliding window and first tokens that stay visible, over packed sequences.
//
// Sequence b has nq queries and L keys; query i stands at position p = L - nq + i among the keys and sees key j
// when j <= p + right and (j >= p - left or j < sinks); a negative left or right is no bound.
// o = sum_j softmax_j(scale q.k_j) v_j over the visible keys; a query that sees none gets zeros.
// A key that a query does not see takes no part in its result, whatever its key and value hold.
#pragma once
#include "rotary.cuh"

namespace gnn {

struct AttendParams {
  HeadsView q, k, v, out;
  const int* q_start;                // [n_seqs + 1]
  const int* kv_start;               // [n_seqs], or null: q_start
  const int* kv_len;                 // [n_seqs], or null: as many as queries
  int n_q_rows, n_kv_rows, n_seqs;
  int max_q;                         // queries of a sequence, at most
  int heads, kv_heads, dim;
  int left, right, sinks;
  float scale_log2;                  // scale * log2(e)
  uint32_t* err;
};

struct Sequence { int q0, nq, k0, len; };

// A sequence's rows, cut to the arrays; *bad when they were not inside.
__device__ __forceinline__ Sequence sequence(const AttendParams& p, int b, bool* bad) {
  Sequence s;
  int q1;
  s.q0 = p.q_start[b];
  q1 = p.q_start[b + 1];
  s.k0 = p.kv_start ? p.kv_start[b] : s.q0;
  s.len = p.kv_len ? p.kv_len[b] : q1 - s.q0;
  *bad = s.q0 < 0 || q1 < s.q0 || q1 > p.n_q_rows || s.len < 0 || s.k0 < 0 || (int64_t)s.k0 + s.len > p.n_kv_rows;
  if (*bad) {
    s.q0 = min(max(s.q0, 0), p.n_q_rows);
    q1 = min(max(q1, s.q0), p.n_q_rows);
    s.k0 = min(max(s.k0, 0), p.n_kv_rows);
    s.len = min(max(s.len, 0), p.n_kv_rows - s.k0);
  }
  s.nq = q1 - s.q0;
  return s;
}

// Keys that the query at position pos sees: [0, first) and [lo, hi), first <= lo.
struct Seen { int first, lo, hi; };
__device__ __forceinline__ Seen seen_keys(int pos, int len, int left, int right, int sinks) {
  Seen s;
  s.hi = right < 0 ? len : (int)max((int64_t)0, min((int64_t)len, (int64_t)pos + right + 1));
  s.lo = left < 0 ? 0 : (int)min((int64_t)s.hi, max((int64_t)0, (int64_t)pos - left));
  s.first = min(sinks, s.lo);
  return s;
}

// One query row of one head by one warp: 32 keys at a time, a key to a lane for the scores, the head's
// elements spread over the lanes for the values.  q: the row in fp32, in shared memory.
template <typename T>
__device__ __noinline__ void attend_row(const AttendParams& p, const Sequence& sq, int i, int head, const float* q) {
  const int lane = threadIdx.x & 31, kv = head / (p.heads / p.kv_heads);
  const Seen s = seen_keys(sq.len - sq.nq + i, sq.len, p.left, p.right, p.sinks);
  const int n = s.first + (s.hi - s.lo);
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int base = 0; base < n; base += 32) {
    const int c = base + lane, j = c < s.first ? c : s.lo + (c - s.first);
    float x = -INFINITY;
    if (c < n) {
      const char* row = p.k.data + (int64_t)(sq.k0 + j) * p.k.row_bytes + kv * p.k.head_bytes;
      x = 0.f;
      for (int d = 0; d < p.dim; d += 8) {
        const Pack<T, 8> k = *reinterpret_cast<const Pack<T, 8>*>(row + d * sizeof(T));
#pragma unroll
        for (int e = 0; e < 8; ++e) x = fmaf(q[d + e], to_f(k.v[e]), x);
      }
      x *= p.scale_log2;
    }
    float top = x;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn;
    const float shrink = exp2f(m - ref), w = c < n ? exp2f(x - ref) : 0.f;
    m = mn;
    l = l * shrink + w;
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] *= shrink;
    for (int r = 0; r < min(32, n - base); ++r) {
      const float wr = __shfl_sync(0xffffffffu, w, r);
      const int jr = __shfl_sync(0xffffffffu, j, r);
      const T* row = reinterpret_cast<const T*>(p.v.data + (int64_t)(sq.k0 + jr) * p.v.row_bytes + kv * p.v.head_bytes);
#pragma unroll
      for (int d = 0; d < 4; ++d)
        if (lane + 32 * d < p.dim) o[d] = fmaf(wr, to_f(row[lane + 32 * d]), o[d]);
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
