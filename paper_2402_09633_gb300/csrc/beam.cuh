// The choice of the best continuations of several hypotheses (beams), and moving the hypotheses' states.
//
// value(b, t) = score[b] + x[b, t] - log sum_t exp(x[b, t]) for the hypotheses b of a group and all t; the `best` largest
// of a group in order, ties to the lowest b * vocab + t.  A hypothesis that has ended has one continuation, its score.
//
// Within a row the order is that of x, so one pass over the logits finds a row's candidates beside its sum: a warp has a
// stretch of a row, a running maximum and sum to a lane, and a list of the elements above the stretch's best-th so far, with
// no barrier between warps until the end.  A second kernel joins the lists row by row, then the rows by value in 64 bits,
// so that rounding neither makes nor breaks ties.  Bound by HBM: logits are read once.
#pragma once
#include "attend_ptx.cuh"
#include "rotary.cuh"

namespace gnn {

constexpr int kBeamMost = 64;        // hypotheses of a group, and continuations that are kept
constexpr int kStripThreads = 256;
constexpr int kStripsMost = 32;      // strips of a row: one to a lane of the warp that joins them
constexpr int kWarpBuffer = 128;     // keys that a warp collects before it keeps the best

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

// How many keys of a list in falling order, `n` of them, are above k.
__device__ __forceinline__ int above(const uint64_t* list, int n, uint64_t k) {
  int a = 0, z = n;
  while (a < z) {
    const int mid = (a + z) / 2;
    if (list[mid] > k) a = mid + 1; else z = mid;
  }
  return a;
}

// A warp's best keys so far.
struct WarpList {
  uint64_t* buf;                     // [kWarpBuffer], the warp's own
  int have;
  float tau;                         // later elements count only above it
};

// Leaves the best keys in order, and the threshold at the last of them.  Keys differ: a key's place is how many are larger.
template <int SLOTS>
__device__ __forceinline__ void warp_rank(WarpList& l, int best) {
  const int lane = threadIdx.x & 31;
  uint64_t k[SLOTS];
  int rank[SLOTS];
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    k[i] = lane + 32 * i < l.have ? l.buf[lane + 32 * i] : 0;
    rank[i] = 0;
  }
#pragma unroll 4
  for (int j = 0; j < l.have; ++j) {
    const uint64_t y = l.buf[j];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) rank[i] += y > k[i];
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < SLOTS; ++i)
    if (lane + 32 * i < l.have && rank[i] < best) l.buf[rank[i]] = k[i];
}
__device__ __noinline__ void warp_prune(WarpList& l, int best) {
  __syncwarp();
  if (l.have <= 32) warp_rank<1>(l, best); else warp_rank<kWarpBuffer / 32>(l, best);
  __syncwarp();
  l.have = min(l.have, best);
  if (l.have == best) l.tau = unordered((uint32_t)(l.buf[best - 1] >> 32));
}

// 2^n for a whole number that is not positive, exactly; zero where that is below what floats hold.
__device__ __forceinline__ float power2(float n) { return n < -126.f ? 0.f : __int_as_float(((int)n + 127) << 23); }

constexpr int kStripPieces = 4;      // of 16 bytes, that a lane takes at a time
constexpr int kStripStages = 3;
constexpr int kStripStage = (32 * kStripPieces + 1) * 16;       // and the one that rows which start between two reach into
constexpr int kStripSmem = kStripThreads / 32 * kStripStages * kStripStage;

template <typename T>
__global__ void __launch_bounds__(kStripThreads, 3) beam_strip_kernel(const __grid_constant__ BeamParams p) {
  constexpr int VEC = 16 / sizeof(T), P = kStripPieces, N = P * VEC, WARPS = kStripThreads / 32;     // elements of a piece, of a lane at a time
  // log2 e in two pieces: the logarithm of a row's sum is to be good to 10^-8 or so, as rows' values are compared with each
  // other.  Sums are relative to 2^r with a whole number r, so that joining them rounds nothing.
  constexpr float kHi = 1.44269504f, kLo = (float)(1.4426950408889634 - (double)1.44269504f);
  extern __shared__ __align__(16) uint8_t strip_smem[];
  __shared__ uint64_t buf_s[WARPS][kWarpBuffer];
  __shared__ float high_s[WARPS];
  __shared__ double sum_s[WARPS];
  __shared__ int have_s[WARPS], count_s[WARPS];
  __shared__ unsigned tau_s;                         // the highest of the warps' thresholds, as it is ordered
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, best = p.best;
  const int row = p.strips == 1 ? (int)blockIdx.x : (int)(blockIdx.x / (unsigned)p.strips);
  const int strip = (int)blockIdx.x - row * p.strips;
  if (tid == 0) tau_s = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  if (p.ended && p.ended[row]) return;
  const T* x = static_cast<const T*>(p.x) + row * p.stride;
  // Pieces by the elements' numbers: rows that hold the same have the same sum to the last bit, wherever in memory they start, so
  // that values which are equal compare so.  Those below `whole`, and not the first of a row that starts between two, come through
  // shared memory, kStripStages rounds ahead of their use; the others element by element.
  const int skew = (int)((uintptr_t)x / sizeof(T) % VEC), bytes = skew * (int)sizeof(T), vocab = p.vocab;
  const int pieces = (vocab + VEC - 1) / VEC, whole = skew == 0 ? vocab / VEC : (vocab + skew) / VEC - 1;
  const int per = (pieces + p.strips * WARPS - 1) / (p.strips * WARPS), p0 = min(pieces, (strip * WARPS + warp) * per),
            p1 = min(pieces, p0 + per);
  const uint4* wide = reinterpret_cast<const uint4*>(x - skew);
  uint8_t* ring = strip_smem + warp * kStripStages * kStripStage;
  // 16 bytes that lie in the row whole: pieces of memory first .. last - 1
  const int first = skew ? 1 : 0, last = (int)(((int64_t)vocab + skew) / VEC);
  auto fetch = [&](int c0, int stage) {              // pieces of memory c0 .. c0 + 32 P
    uint8_t* to = ring + stage * kStripStage;
    if (c0 < p1) {
#pragma unroll
      for (int h = 0; h <= P; ++h) {
        const int i = h * 32 + lane, at = c0 + i;
        if (i <= 32 * P && at >= first && at < last && at <= p1)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to + i * 16)), "l"(wide + at) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  float m = -INFINITY, r = 0.f, s = 0.f;
  WarpList list = {buf_s[warp], 0, -INFINITY};
  const int spare = kWarpBuffer - 32;                // keys that leave room for those of another element of all lanes
  const int enough = min(spare, max(32, 2 * best));  // keys from which on a new threshold is worth its price
  volatile unsigned* shared_tau = &tau_s;
#pragma unroll
  for (int k = 0; k < kStripStages - 1; ++k) fetch(p0 + k * 32 * P, k);
  int stage = 0;
  for (int c0 = p0; c0 < p1; c0 += 32 * P) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStripStages - 2) : "memory");
    __syncwarp();                                    // what lies in the stage, and that the one before has been read
    fetch(c0 + (kStripStages - 1) * 32 * P, stage == 0 ? kStripStages - 1 : stage - 1);
    float v[N];
    {
      const uint8_t* from = ring + stage * kStripStage;
      stage = stage + 1 == kStripStages ? 0 : stage + 1;
#pragma unroll
      for (int h = 0; h < P; ++h) {
        const int piece = c0 + h * 32 + lane;
        Pack<T, VEC> k;
        if (piece < min(p1, whole) && piece >= first) {
          const uint4* at = reinterpret_cast<const uint4*>(from) + h * 32 + lane;
          *reinterpret_cast<uint4*>(&k) = skew == 0 ? *at : load_skewed(at, bytes);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) k.v[e] = piece < p1 && (int64_t)piece * VEC + e < vocab ? x[(int64_t)piece * VEC + e] : from_f<T>(-INFINITY);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[h * VEC + e] = to_f(k.v[e]);
      }
    }
    float high = v[0];
#pragma unroll
    for (int e = 1; e + 1 < N; e += 2) high = max3(high, v[e], v[e + 1]);
    high = fmaxf(high, v[N - 1]);
    if (high > m) {
      const float to = ceilf(high * kHi);
      if (m > -INFINITY) s *= power2(r - to);
      m = high;
      r = to;
    }
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float2 y = make_float2(v[e], v[e + 1]);
      const float2 z = __ffma2_rn(y, make_float2(kLo, kLo), __ffma2_rn(y, make_float2(kHi, kHi), make_float2(-r, -r)));
      sum[e >> 1 & 1] = __fadd2_rn(sum[e >> 1 & 1], make_float2(exp2_approx(z.x), exp2_approx(z.y)));
    }
    s += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
    // candidates: later elements of the same value as the threshold lose the tie
    if (!__any_sync(0xffffffffu, high > list.tau)) continue;
    // of these elements, those above the threshold and from here on: another warp's threshold bounds the block's best from
    // below too, but elements equal to it may have lower numbers than that warp's
    const unsigned theirs = *shared_tau;
    float from = theirs ? unordered(theirs) : -INFINITY;
    if (!__any_sync(0xffffffffu, high >= from)) continue;
    if (list.tau == -INFINITY && theirs == 0) {
      // at first as many lanes' largest elements bound the best from below, or all lanes' two largest
      if (best <= 32) {
        int rank = 0;
#pragma unroll
        for (int d = 0; d < 32; ++d) {
          const float y = __shfl_sync(0xffffffffu, high, d);
          rank += y > high || (y == high && d < lane);
        }
        from = __shfl_sync(0xffffffffu, high, __ffs(__ballot_sync(0xffffffffu, rank == best - 1)) - 1);
      } else {
        float a = -INFINITY, z = -INFINITY;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          z = fmaxf(z, fminf(a, v[e]));
          a = fmaxf(a, v[e]);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) z = fminf(z, __shfl_xor_sync(0xffffffffu, z, d));
        from = z;
      }
    }
    auto count = [&] {
      int n = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) n += v[e] > list.tau && v[e] >= from;
      return n;
    };
    auto append = [&](int at) {                      // in any order: keys differ
#pragma unroll
      for (int h = 0; h < P; ++h)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float y = v[h * VEC + e];
          if (y > list.tau && y >= from) list.buf[at++] = beam_key(y, (uint32_t)((c0 + h * 32 + lane) * VEC + e));
        }
    };
    const int mine = count(), more = __reduce_add_sync(0xffffffffu, mine);
    if (list.have + more <= kWarpBuffer) {
      if (lane == 0) count_s[warp] = list.have;
      __syncwarp();
      if (mine) append(atomicAdd(&count_s[warp], mine));
      list.have += more;
    } else {                                         // rows that rise, or are all the same: lane by lane
#pragma unroll 1
      for (int d = 0; d < 32; ++d) {
        const int now = __shfl_sync(0xffffffffu, count(), d);
        if (now == 0) continue;
        if (list.have > spare) {
          // The threshold is of elements with any numbers then: what is left of this round counts from it on.
          const float before = list.tau;
          warp_prune(list, best);
          from = fmaxf(from, list.tau);
          list.tau = before;
          --d;
          continue;
        }
        if (lane == d) append(list.have);
        list.have += now;
      }
    }
    __syncwarp();
    if (list.have >= enough || (list.tau == -INFINITY && list.have >= best)) {
      warp_prune(list, best);
      if (lane == 0 && list.have == best) atomicMax(&tau_s, ordered(list.tau));
    }
  }
  warp_prune(list, best);
  if (lane == 0) have_s[warp] = list.have;
  // the threads' sums
  float high = m == -INFINITY ? -INFINITY : r;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, d));
  if (lane == 0) high_s[warp] = high;
  __syncthreads();
  high = high_s[0];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) high = fmaxf(high, high_s[w]);
  // (a power of two below what floats hold is below what counts, and an infinite r has made s NaN)
  double sum = s == 0.f ? 0. : (double)(s * power2(r - (high == -INFINITY ? 0.f : high)));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) sum_s[warp] = sum;
  // the warps' lists: a key's place is its own and what the others have above it
  uint64_t* out = p.lists + (int64_t)blockIdx.x * best;
  int all = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) all += have_s[w];
  for (int i = lane; i < list.have; i += 32) {
    const uint64_t k = list.buf[i];
    int rank = i;
#pragma unroll
    for (int w = 0; w < WARPS; ++w)
      if (w != warp) rank += above(buf_s[w], have_s[w], k);
    if (rank < best) out[rank] = k;
  }
  for (int i = all + tid; i < best; i += kStripThreads) out[i] = 0;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < WARPS; ++w) sum += sum_s[w];
    p.sums[blockIdx.x] = {sum, high};
  }
}

constexpr int kJoinThreads = 256;

// One group to a block: first the strips of every row, then the rows, each time a candidate's place being how many of the
// other lists' are before it.
__global__ void __launch_bounds__(kJoinThreads) beam_join_kernel(const __grid_constant__ BeamParams p) {
  extern __shared__ __align__(16) uint64_t join_smem[];
  __shared__ double base_s[kBeamMost];               // a row's sum; then what is added to a logit
  __shared__ float top_s[kBeamMost];
  __shared__ int taken_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, best = p.best, beams = p.beams, strips = p.strips;
  const int64_t group = blockIdx.x, row0 = group * beams;
  uint64_t* rows = join_smem;                        // [beams][best]
  uint64_t* values = rows + beams * best;            // the same, as they are ordered: comparing 64-bit floats takes long here
  uint64_t* lists = values + beams * best;           // [warps][strips][best]
  if (tid == 0) taken_s = 0;
  pdl_wait();
  for (int b = warp; b < beams; b += kJoinThreads / 32) {
    const int64_t row = row0 + b;
    const bool ended = p.ended && p.ended[row];
    uint64_t* mine = rows + b * best;
    if (ended) {
      for (int i = lane; i < best; i += 32) mine[i] = i == 0 ? beam_key(0.f, (uint32_t)p.end) : 0;
      if (lane == 0) {
        base_s[b] = 1.;
        top_s[b] = 0.f;
      }
    } else {
      const BeamSum part = lane < strips ? p.sums[row * strips + lane] : BeamSum{0., -INFINITY};
      const uint64_t* from = p.lists + row * strips * best;
      uint64_t* to = strips == 1 ? mine : lists + warp * strips * best;
      for (int i = lane; i < strips * best; i += 32) to[i] = from[i];
      float top = part.r;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      double sum = part.s == 0. ? 0. : part.s * (double)power2(part.r - (top == -INFINITY ? 0.f : top));
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (lane == 0) {
        base_s[b] = sum;
        top_s[b] = top;
      }
      __syncwarp();
      if (strips > 1) {
        for (int i = lane; i < best; i += 32) mine[i] = 0;
        __syncwarp();
        for (int i = lane; i < strips * best; i += 32) {
          const uint64_t k = to[i];
          if (k == 0) continue;
          const int s = i / best;
          int rank = i - s * best;
          for (int t = 0; t < strips && rank < best; ++t)
            if (t != s) rank += above(to + t * best, best, k);
          if (rank < best) mine[rank] = k;
        }
        __syncwarp();
      }
    }
  }
  __syncthreads();
  // 64-bit arithmetic is slow here: one logarithm for all rows
  if (tid < beams) base_s[tid] = (double)p.score[row0 + tid] - ((double)top_s[tid] + log2(base_s[tid])) * 0.6931471805599453;
  __syncthreads();
  for (int i = tid; i < beams * best; i += kJoinThreads) {
    const uint64_t k = rows[i];
    const double v = k ? base_s[i / best] + (double)unordered((uint32_t)(k >> 32)) : -INFINITY;
    const uint64_t u = (uint64_t)__double_as_longlong(v + 0.);
    values[i] = !(v > -INFINITY) ? 0 : u >> 63 ? ~u : u | 1ull << 63;        // 0: none, or NaN
  }
  __syncthreads();
  int taken = 0;
  for (int i = tid; i < beams * best; i += kJoinThreads) {
    const uint64_t v = values[i];
    if (v == 0) continue;
    const int b = i / best;
    int rank = i - b * best;
    for (int c = 0; c < beams && rank < best; ++c) {
      if (c == b) continue;
      const uint64_t* list = values + c * best;      // falling; of equal values those of lower rows come first
      int a = 0, z = best;
      while (a < z) {
        const int mid = (a + z) / 2;
        if (c < b ? list[mid] >= v : list[mid] > v) a = mid + 1; else z = mid;
      }
      rank += a;
    }
    if (rank >= best) continue;
    const int64_t o = group * best + rank;
    p.out_score[o] = (float)__longlong_as_double((long long)(v >> 63 ? v & ~(1ull << 63) : ~v));
    p.out_parent[o] = b;
    p.out_token[o] = (int)~(uint32_t)rows[i];
    ++taken;
  }
  atomicAdd(&taken_s, taken);
  __syncthreads();
  for (int i = taken_s + tid; i < best; i += kJoinThreads) {
    const int64_t o = group * best + i;
    p.out_score[o] = -INFINITY;
    p.out_parent[o] = 0;
    p.out_token[o] = -1;
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
