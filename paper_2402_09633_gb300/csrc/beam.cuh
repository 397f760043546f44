// The choice of the best continuations of several hypotheses (beams), and moving the hypotheses' states.
//
// value(b, t) = score[b] + x[b, t] - log sum_t exp(x[b, t]) for the hypotheses b of a group and all t; the `best` largest
// of a group in order, ties to the lowest b * vocab + t.  A hypothesis that has ended has one continuation, its score.
//
// Within a row the order is that of x, so one pass over the logits finds a row's candidates beside its sum: a block
// has a strip of a row, keeps a running maximum and sum to a thread, and a list of the elements above the strip's best-th
// so far.  A second kernel joins the strips row by row, then the rows by value in 64 bits, so that rounding
// neither makes nor breaks ties.  Bound by HBM: logits are read once.
#pragma once
#include "attend_ptx.cuh"
#include "rotary.cuh"

namespace gnn {

constexpr int kBeamMost = 64;        // hypotheses of a group, and continuations that are kept
constexpr int kStripThreads = 256;
constexpr int kStripsMost = 32;      // strips of a row: one to a lane of the warp that joins them

struct alignas(16) BeamSum { double s; float r; };    // the sum of 2^(x log2 e - r) over a strip
struct BeamParams {
  const void* x;                     // [groups * beams, vocab]
  int64_t stride;                    // elements
  const float* score;                // [groups * beams]
  const uint8_t* ended;              // [groups * beams], or null
  int end, beams, vocab, best, strips;
  int64_t rows;                      // groups * beams
  BeamSum* sums;                     // [rows * strips]
  uint64_t* lists;                   // [rows * strips][best]: its largest elements as keys, in order; 0: none
  float* out_score;                  // [groups * best]
  int *out_parent, *out_token;
};

// Keys in the order of elements: the larger x, then the lower index.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);       // -0 as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint64_t beam_key(float x, uint32_t index) { return (uint64_t)ordered(x) << 32 | ~index; }

// 16 bytes from `bytes` (1..15) past an aligned address on, out of the two aligned pieces that hold them.
__device__ __forceinline__ uint4 load_skewed(const void* at, int bytes) {
  const uint4 a = *static_cast<const uint4*>(at), b = static_cast<const uint4*>(at)[1];
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (bytes & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (bytes & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const int bits = (bytes & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}

template <typename T>
__global__ void __launch_bounds__(kStripThreads) beam_strip_kernel(const __grid_constant__ BeamParams p) {
  constexpr int VEC = 16 / sizeof(T), N = 2 * VEC;   // elements of 16 bytes; of a thread at a time
  constexpr int CHUNK = kStripThreads * N, CAP = CHUNK + 256;
  // log2 e in two pieces, and sums relative to 2^r with r as it is rounded: the logarithm of a row's sum is to be good
  // to 10^-8 or so, as rows' values are compared with each other
  constexpr float kHi = 1.44269504f, kLo = (float)(1.4426950408889634 - (double)1.44269504f);
  __shared__ uint64_t buf[CAP], pick_s[kBeamMost], top_s[kBeamMost];
  __shared__ int count_s;
  __shared__ float high_s[kStripThreads / 32];
  __shared__ double sum_s[kStripThreads / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t row = blockIdx.x / p.strips;
  const int strip = (int)(blockIdx.x - row * p.strips);
  if (tid == 0) count_s = 0;
  pdl_wait();
  pdl_trigger();
  if (p.ended && p.ended[row]) return;
  const T* x = static_cast<const T*>(p.x) + row * p.stride;
  // Pieces of 16 bytes, by the elements' numbers: rows that hold the same have the same sum to the last bit, wherever in
  // memory they start, so that values which are equal compare so.
  const int skew = (int)((uintptr_t)x / sizeof(T) % VEC);
  const int64_t pieces = ((int64_t)p.vocab + VEC - 1) / VEC;
  const int64_t per = (pieces + p.strips - 1) / p.strips;
  const int64_t p0 = min(pieces, strip * per), p1 = min(pieces, p0 + per);
  __syncthreads();

  float m = -INFINITY, r = 0.f, s = 0.f, tau = -INFINITY;
  int have = 0;                                      // keys in buf, as every thread knows it
  // Leaves the best keys of buf in order in its first places, and the threshold at the last of them.
  auto prune = [&] {
    int n = have;
    uint64_t least = 0;
    if (n > kStripThreads) {                         // the largest key that `best` of them reach, bit by bit
#pragma unroll 1
      for (int bit = 63; bit >= 0; --bit) {
        const uint64_t t = least | 1ull << bit;
        int c = 0;
        for (int i = tid; i < n; i += kStripThreads) c += buf[i] >= t;
        c = __reduce_add_sync(0xffffffffu, c);
        if (tid == 0) count_s = 0;
        __syncthreads();
        if (lane == 0) atomicAdd(&count_s, c);
        __syncthreads();
        if (count_s >= p.best) least = t;
        __syncthreads();
      }
    }
    const uint64_t* from = buf;
    if (n > kStripThreads) {
      if (tid == 0) count_s = 0;
      __syncthreads();
      for (int i = tid; i < n; i += kStripThreads)
        if (buf[i] >= least) pick_s[atomicAdd(&count_s, 1)] = buf[i];
      __syncthreads();
      from = pick_s;
      n = p.best;
    }
    if (tid < n) {                                   // keys differ: as many come before one as are larger
      const uint64_t k = from[tid];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += from[j] > k;
      if (rank < p.best) top_s[rank] = k;
    }
    __syncthreads();
    have = min(n, p.best);
    if (tid < have) buf[tid] = top_s[tid];
    if (tid == 0) count_s = have;
    if (have == p.best) tau = unordered((uint32_t)(top_s[have - 1] >> 32));
    __syncthreads();
  };

  for (int64_t c0 = p0; c0 < p1; c0 += 2 * kStripThreads) {
    float v[N];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t piece = c0 + h * kStripThreads + tid, e0 = piece * VEC;
      Pack<T, VEC> k;
      if (piece < p1 && (skew == 0 ? e0 + VEC <= p.vocab : piece > 0 && e0 + 2 * VEC - skew <= p.vocab)) {
        *reinterpret_cast<uint4*>(&k) = skew == 0 ? __ldcs(reinterpret_cast<const uint4*>(x + e0)) : load_skewed(x + e0 - skew, skew * (int)sizeof(T));
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) k.v[e] = piece < p1 && e0 + e < p.vocab ? x[e0 + e] : from_f<T>(-INFINITY);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[h * VEC + e] = to_f(k.v[e]);
    }
    float high = v[0];
#pragma unroll
    for (int e = 1; e < N; ++e) high = fmaxf(high, v[e]);
    if (high > m) {
      const float next = high * kHi;
      if (m > -INFINITY) s *= exp2_approx(r - next);
      m = high;
      r = next;
    }
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float2 y = make_float2(v[e], v[e + 1]);
      const float2 z = __ffma2_rn(y, make_float2(kLo, kLo), __ffma2_rn(y, make_float2(kHi, kHi), make_float2(-r, -r)));
      sum = __fadd2_rn(sum, make_float2(exp2_approx(z.x), exp2_approx(z.y)));
    }
    s += sum.x + sum.y;
    // candidates: later elements of the same value as the threshold lose the tie
    if (!__syncthreads_or(high > tau)) continue;
    float least = tau;                               // of this chunk's, those above it, or from it on
    bool from = false;
    int mine = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) mine += v[e] > tau;
    if (__syncthreads_count(mine > 0) >= p.best) {
      // `best` threads' largest elements bound the strip's best-th from below
      uint32_t t = 0;
      const uint32_t h = high > tau ? ordered(high) : 0;
#pragma unroll 1
      for (int bit = 31; bit >= 0; --bit)
        if (__syncthreads_count(h >= (t | 1u << bit)) >= p.best) t |= 1u << bit;
      least = unordered(t);
      from = true;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float y = v[h * VEC + e];
        if (y > tau && (from ? y >= least : y > least))
          buf[atomicAdd(&count_s, 1)] = beam_key(y, (uint32_t)((c0 + h * kStripThreads + tid) * VEC + e));
      }
    __syncthreads();
    have = count_s;
    __syncthreads();
    if (have > 256 || tau == -INFINITY) prune();
  }
  if (have > 0) prune();
  uint64_t* list = p.lists + (int64_t)blockIdx.x * p.best;
  if (tid < p.best) list[tid] = tid < have ? buf[tid] : 0;
  // the threads' sums
  float high = m == -INFINITY ? -INFINITY : r;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, d));
  if (lane == 0) high_s[warp] = high;
  __syncthreads();
  high = high_s[0];
  for (int w = 1; w < kStripThreads / 32; ++w) high = fmaxf(high, high_s[w]);
  double sum = s == 0.f ? 0. : (double)(s * exp2f(r - (high == -INFINITY ? 0.f : high)));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) sum_s[warp] = sum;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kStripThreads / 32; ++w) sum += sum_s[w];
    p.sums[blockIdx.x] = {sum, high};
  }
}

constexpr int kJoinWarps = 8;

// One group to a block: a warp joins the strips of a row at a time, the first warp joins the rows.
__global__ void __launch_bounds__(32 * kJoinWarps) beam_join_kernel(const __grid_constant__ BeamParams p) {
  __shared__ uint64_t list_s[kBeamMost][kBeamMost];  // [hypothesis][rank]
  __shared__ double base_s[kBeamMost];               // what is added to a logit
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t group = blockIdx.x;
  pdl_wait();
  for (int b = warp; b < p.beams; b += kJoinWarps) {
    const int64_t row = group * p.beams + b;
    const float score = p.score[row];
    if (p.ended && p.ended[row]) {
      for (int i = lane; i < p.best; i += 32) list_s[b][i] = i == 0 ? beam_key(0.f, (uint32_t)p.end) : 0;
      if (lane == 0) base_s[b] = (double)score;
      continue;
    }
    const BeamSum part = lane < p.strips ? p.sums[row * p.strips + lane] : BeamSum{0., -INFINITY};
    float top = part.r;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    double sum = part.s == 0. ? 0. : part.s * exp2((double)part.r - (double)top);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) base_s[b] = (double)score - ((double)top + log2(sum)) * 0.6931471805599453;
    // the strips' lists, each in order, into one
    const uint64_t* list = p.lists + (row * p.strips + lane) * p.best;
    int at = 0;
    uint64_t head = lane < p.strips ? list[0] : 0;
    for (int i = 0; i < p.best; ++i) {
      uint64_t k = head;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) k = max(k, __shfl_xor_sync(0xffffffffu, k, d));
      if (lane == 0) list_s[b][i] = k;
      if (k != 0 && head == k) head = ++at < p.best ? list[at] : 0;
    }
  }
  __syncthreads();
  if (warp != 0) return;
  // rows lane and lane + 32
  int at[2] = {0, 0};
  uint64_t key[2];
  double value[2];
  auto fetch = [&](int h) {
    const int b = lane + 32 * h;
    key[h] = b < p.beams && at[h] < p.best ? list_s[b][at[h]] : 0;
    value[h] = key[h] ? base_s[b] + (double)unordered((uint32_t)(key[h] >> 32)) : -INFINITY;
    if (!(value[h] > -INFINITY)) {                   // none, or NaN
      value[h] = -INFINITY;
      key[h] = 0;
    }
  };
  fetch(0);
  fetch(1);
  for (int i = 0; i < p.best; ++i) {
    double v = value[0];
    uint64_t k = key[0];
    int b = lane;
    if (value[1] > v) { v = value[1]; k = key[1]; b = lane + 32; }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const double v2 = __shfl_xor_sync(0xffffffffu, v, d);
      const uint64_t k2 = __shfl_xor_sync(0xffffffffu, k, d);
      const int b2 = __shfl_xor_sync(0xffffffffu, b, d);
      if (v2 > v || (v2 == v && b2 < b)) { v = v2; k = k2; b = b2; }
    }
    if (lane == 0) {
      const int64_t o = group * p.best + i;
      const bool none = v == -INFINITY;
      p.out_score[o] = (float)v;
      p.out_parent[o] = none ? 0 : b;
      p.out_token[o] = none ? -1 : (int)~(uint32_t)k;
    }
    if (v > -INFINITY && b % 32 == lane) {
      const int h = b / 32;
      if (h == 0) { ++at[0]; fetch(0); } else { ++at[1]; fetch(1); }
    }
  }
}

// ------------------------------------------------------------------ states
// Rows of hypotheses moved to those that continue them: slot i of a group gets what slot parent[i] of the group held.
// A thread has a column of a few bytes of all slots of a group: it fetches what any slot needs, through shared memory
// places of its own, and then writes, so states are moved in place without a second buffer or a barrier.  A column
// is read once for each different parent, however many continue it.  Bound by HBM.
constexpr int kMoveThreads = 128;
constexpr int kMoveStates = 16;      // of a launch

struct MoveState {
  char* data;
  char* out;                         // data: in place
  int64_t stride, out_stride, bytes; // of a row
  int width;                         // bytes of a column: 16, 4 or 1
};
struct MovePages {                   // keys or values in pages: the open page's rows
  char* data;
  int64_t row_bytes, head_bytes;
  int heads, width;
};
struct MoveParams {
  const int* parent;                 // [groups * beams]
  int64_t groups;
  int beams, states, pools, segments, dim_bytes;
  MoveState state[kMoveStates];
  MovePages pool[kMoveStates];
  int* table;                        // the paged form's; [groups * beams] rows
  const int* kv_len;
  int64_t table_stride, n_pages;
  int table_width, shift;
  uint32_t* err;
};

template <int W> struct MoveWord;
template <> struct MoveWord<16> { using type = uint4; };
template <> struct MoveWord<4> { using type = uint32_t; };
template <> struct MoveWord<1> { using type = uint8_t; };

// Columns [c0, n) in steps of `step`: from(c) and to(c) give a column's address in slot 0.. of the group, by slot.
template <int W, typename From, typename To>
__device__ __forceinline__ void move_columns(int64_t c0, int64_t n, int64_t step, int beams, const int8_t* parent, uint64_t need,
                                             uint64_t get, uint8_t* mine, From from, To to) {
  using Word = typename MoveWord<W>::type;
  for (int64_t c = c0; c < n; c += step) {
    for (uint64_t b = need; b; b &= b - 1) {
      const int i = __ffsll((long long)b) - 1;
      uint8_t* dst = mine + i * (kMoveThreads * W);
      if constexpr (W == 1) {
        *dst = *reinterpret_cast<const uint8_t*>(from(i, c));
      } else {
        if constexpr (W == 16)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(from(i, c)) : "memory");
        else
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(from(i, c)) : "memory");
      }
    }
    if constexpr (W > 1) asm volatile("cp.async.wait_all;" ::: "memory");
    for (uint64_t b = get; b; b &= b - 1) {
      const int i = __ffsll((long long)b) - 1;
      *reinterpret_cast<Word*>(to(i, c)) = *reinterpret_cast<const Word*>(mine + parent[i] * (kMoveThreads * W));
    }
  }
}

// Blocks: segment by segment of a group of a state or pool (the last: the table).
__global__ void __launch_bounds__(kMoveThreads) beam_move_kernel(const __grid_constant__ MoveParams p) {
  extern __shared__ __align__(16) uint8_t move_smem[];
  __shared__ int8_t parent_s[kBeamMost];
  __shared__ int entry_s[kBeamMost];
  __shared__ unsigned long long need_s, get_s;
  __shared__ int len_s, uneven_s, bad_s;
  const int tid = threadIdx.x;
  const int64_t per = (int64_t)p.segments * p.groups;
  const int what = (int)(blockIdx.x / per);
  const int64_t rest = blockIdx.x - what * per, group = rest / p.segments, first = group * p.beams;
  const int segment = (int)(rest - group * p.segments);
  const bool paged = p.table != nullptr;
  if (tid == 0) need_s = get_s = 0, uneven_s = bad_s = 0;
  pdl_wait();
  if (tid == 0 && paged) len_s = p.kv_len[first];
  __syncthreads();
  const bool in_place = paged || p.state[what].out == p.state[what].data;
  if (tid < p.beams) {
    int a = p.parent[first + tid];
    if (a < 0 || a >= p.beams) {
      if (paged) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
      a = tid;
    }
    parent_s[tid] = (int8_t)a;
    if (!in_place || a != tid) {
      atomicOr(&need_s, 1ull << a);
      atomicOr(&get_s, 1ull << tid);
    }
    if (paged && p.kv_len[first + tid] != len_s) uneven_s = 1;
  }
  __syncthreads();
  const uint64_t need = need_s, get = get_s;
  if (get == 0) return;
  const int64_t c0 = (int64_t)segment * kMoveThreads + tid, step = (int64_t)p.segments * kMoveThreads;
  if (!paged) {
    const MoveState& s = p.state[what];
    const char* src = s.data + first * s.stride;
    char* dst = s.out + first * s.out_stride;
    auto go = [&](auto w) {
      constexpr int W = decltype(w)::value;
      move_columns<W>(c0, s.bytes / W, step, p.beams, parent_s, need, get, move_smem + tid * W,
                      [&](int i, int64_t c) { return src + i * s.stride + c * W; },
                      [&](int i, int64_t c) { return dst + i * s.out_stride + c * W; });
    };
    if (s.width == 16) go(std::integral_constant<int, 16>());
    else if (s.width == 4) go(std::integral_constant<int, 4>());
    else go(std::integral_constant<int, 1>());
    return;
  }
  const int len = len_s, full = len >> p.shift, part = len & ((1 << p.shift) - 1);
  if (uneven_s || len < 0 || full > p.table_width || (full == p.table_width && part > 0)) {
    if (tid == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
    return;
  }
  if (part > 0 && tid < p.beams) {                   // the open page of each slot; nothing writes its entry
    const int e = p.table[(first + tid) * p.table_stride + full];
    entry_s[tid] = e;
    if (e < 0 || e >= p.n_pages) bad_s = 1;
  }
  __syncthreads();
  if (bad_s) {
    if (tid == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
    return;
  }
  if (what == p.pools) {                             // entries of full pages
    int* t = p.table + first * p.table_stride;
    move_columns<4>(c0, full, step, p.beams, parent_s, need, get, move_smem + tid * 4,
                    [&](int i, int64_t c) { return t + i * p.table_stride + c; },
                    [&](int i, int64_t c) { return t + i * p.table_stride + c; });
    return;
  }
  if (part == 0) return;
  const MovePages& s = p.pool[what];
  auto go = [&](auto w) {
    constexpr int W = decltype(w)::value;
    const unsigned piece = (unsigned)p.dim_bytes / W, row = piece * (unsigned)s.heads;
    auto at = [&](int i, int64_t c) {
      const unsigned r = (unsigned)c / row, in = (unsigned)c - r * row, h = in / piece;
      return s.data + (((int64_t)entry_s[i] << p.shift) + r) * s.row_bytes + (int64_t)h * s.head_bytes + (in - h * piece) * W;
    };
    move_columns<W>(c0, (int64_t)part * row, step, p.beams, parent_s, need, get, move_smem + tid * W, at, at);
  };
  if (s.width == 16) go(std::integral_constant<int, 16>());
  else if (s.width == 4) go(std::integral_constant<int, 4>());
  else go(std::integral_constant<int, 1>());
}

}  // namespace gnn
