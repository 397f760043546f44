// The choice of the best continuations of several hypotheses (beams), and moving the hypotheses' states.
//
// value(b, t) = score[b] + x[b, t] - log sum_t exp(x[b, t]) for the hypotheses b of a group and all t; the `best` largest
// of a group in order, ties to the lowest b * vocab + t.  A hypothesis that has ended has one continuation, its score.
//
// Within a row the order is that of x, so one pass over the logits finds a row's candidates beside its sum: a warp has a
// stretch of a row, a running maximum and sum to a lane, and a sorted list of its best so far in registers; elements
// below the list's last, or below what the block's lists bound the best by, cost a comparison.  A second kernel joins the lists row
// by row, then the rows by value in 64 bits, so that rounding neither makes nor breaks ties.
//
// Logits are read once: bound by HBM where rows are long (16 groups of 16 rows of 300,000 fp32: 67 us, 4.6 TB/s with the join's
// 8 us; the floor is 45), by instructions where they are short (64 groups of 8 rows of 32,003 bf16: 29 us, issue 61 %; half of it first
// lists and candidates), by the chain of both kernels where they are few (4 rows of 1,000: 9 us).
#pragma once
#include "attend_ptx.cuh"
#include <cfloat>
#include "rotary.cuh"

namespace gnn {

constexpr int kBeamMost = 64;        // hypotheses of a group, and continuations that are kept
constexpr float kLog2e = 1.44269504f;
constexpr int kStripThreads = 256, kStripBlocks = 4;         // and blocks to an SM
constexpr int kStripsMost = 32;      // strips of a row: at most one to a lane of the warp that joins them

// A strip's sum of 2^(x log2 e - r); or, where its largest element is `far`, past kBeamFar, of 2^((x - r) log2 e) with r that element.
struct alignas(16) BeamSum { double s; float r; int far; };
// Up to here x log2 e is rounded by 1/16 at most, so that its whole part serves as a reference.
constexpr float kBeamFar = 1048576.f;
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

// A warp's best keys in falling order: place `lane` and, above 32 of them, place 32 + lane.
struct WarpList { uint64_t a, z; };

__device__ __forceinline__ uint64_t exchange(uint64_t k, int d, bool larger) {
  const uint64_t y = __shfl_xor_sync(0xffffffffu, k, d);
  return (y > k) == larger ? y : k;
}
// Keys that rise and then fall over the lanes, or the reverse, in falling order.
__device__ __forceinline__ uint64_t merge_lanes(uint64_t k) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) k = exchange(k, d, (threadIdx.x & d) == 0);
  return k;
}
// A key of every lane in falling order.  (A bitonic network: Batcher 1968.)
__device__ __forceinline__ uint64_t sort_lanes(uint64_t k) {
#pragma unroll
  for (int n = 2; n <= 32; n *= 2)
#pragma unroll
    for (int d = n / 2; d > 0; d >>= 1) k = exchange(k, d, ((threadIdx.x & d) == 0) == ((threadIdx.x & n & 31) == 0));
  return k;
}
// The best of a list and of a key of every lane (0: none).
__device__ __forceinline__ void take_lanes(WarpList& l, uint64_t k, int best) {
  k = __shfl_xor_sync(0xffffffffu, sort_lanes(k), 31);               // rising
  if (best > 32) {
    const uint64_t y = __shfl_xor_sync(0xffffffffu, merge_lanes(max(l.z, k)), 31);
    const uint64_t hi = max(l.a, y), lo = min(l.a, y);
    l.a = merge_lanes(hi);
    l.z = merge_lanes(lo);
  } else {
    l.a = merge_lanes(max(l.a, k));
  }
}
__device__ __forceinline__ uint64_t list_at(const WarpList& l, int i) {
  return __shfl_sync(0xffffffffu, i < 32 ? l.a : l.z, i & 31);
}

// 2^n for a whole number that is not positive, exactly; zero where that is below what floats hold.
__device__ __forceinline__ float power2(float n) { return n < -126.f ? 0.f : __int_as_float(((int)n + 127) << 23); }

constexpr int kStripHeld = 8;         // candidates that are put in a warp's list together, at least
constexpr int kLaneElements = 16;    // that a lane takes at a time
template <typename T> constexpr int strip_stages() { return sizeof(T) == 4 ? 3 : 4; }            // what lets four blocks share an SM
template <typename T> constexpr int strip_pieces() { return kLaneElements * (int)sizeof(T) / 16; }                // of 16 bytes
template <typename T> constexpr int strip_stage() { return (32 * strip_pieces<T>() + 1) * 16; }    // and the one that rows which start between two reach into
template <typename T> constexpr int strip_smem() { return kStripThreads / 32 * strip_stages<T>() * strip_stage<T>(); }

// A thread's share of the sum of 2^((x - top) log2 e) over its block's strip.  Finds the strip by itself, so that the kernel keeps nothing for it.
template <typename T>
__device__ __noinline__ double beam_far_sum(const BeamParams& p, float top) {
  constexpr int VEC = 16 / sizeof(T);
  const int64_t row = blockIdx.x / (unsigned)p.strips, strip = blockIdx.x - row * p.strips;
  const int64_t pieces = ((int64_t)p.vocab + VEC - 1) / VEC, warps = kStripThreads / 32, per = (pieces + p.strips * warps - 1) / (p.strips * warps);
  const int64_t a = strip * warps * per * VEC, z = min((int64_t)p.vocab, a + warps * per * VEC);
  const T* x = static_cast<const T*>(p.x) + row * p.stride;
  double sum = 0.;
  for (int64_t i = a + threadIdx.x; i < z; i += kLaneElements * kStripThreads) {
    float some = 0.f;
#pragma unroll 4
    for (int e = 0; e < kLaneElements; ++e) {
      const int64_t at = i + e * kStripThreads;
      if (at < z) some += exp2_approx((to_f(x[at]) - top) * kLog2e);
    }
    sum += some;
  }
  return sum;
}

template <typename T>
__global__ void __launch_bounds__(kStripThreads, kStripBlocks) beam_strip_kernel(const __grid_constant__ BeamParams p) {
  constexpr int VEC = 16 / sizeof(T), P = strip_pieces<T>(), N = kLaneElements, WARPS = kStripThreads / 32, STAGE = strip_stage<T>(), STAGES = strip_stages<T>();
  // Sums are of 2^(c x - r) with c = log2 e rounded, and their logarithm is divided by c again: that leaves 1.3e-8 of the weights'
  // entropy as an error, where c is off by 1.3e-8.  r is a whole number, so that joining sums rounds nothing.  Finite elements far below
  // zero (masks) have the reference of -kBeamFar, beside which they weigh nothing.  A strip whose largest element is past kBeamFar on either
  // side is summed up once more at its end, with that element taken off before the product is rounded.
  extern __shared__ __align__(16) uint8_t strip_ring[];
  __shared__ uint64_t list_s[WARPS][kBeamMost];      // at first what is held back
  __shared__ float high_s[WARPS];
  __shared__ double sum_s[WARPS];
  __shared__ int have_s[WARPS];
  __shared__ unsigned bound_s[WARPS];                // of each warp's list, the value at place best / 8, as it is ordered
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, best = p.best;
  const int row = p.strips == 1 ? (int)blockIdx.x : (int)(blockIdx.x / (unsigned)p.strips);
  const int strip = (int)blockIdx.x - row * p.strips;
  if (tid < WARPS) bound_s[tid] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  if (p.ended && p.ended[row]) return;
  const T* x = static_cast<const T*>(p.x) + row * p.stride;
  // Pieces by the elements' numbers: rows that hold the same have the same sum to the last bit, wherever in memory they start, so
  // that values which are equal compare so.  Those below `whole`, and not the first of a row that starts between two, come through
  // shared memory, STAGES rounds ahead of their use; the others element by element.
  const int skew = (int)((uintptr_t)x / sizeof(T) % VEC), bytes = skew * (int)sizeof(T), vocab = p.vocab;
  const int pieces = (vocab + VEC - 1) / VEC, whole = skew == 0 ? vocab / VEC : (vocab + skew) / VEC - 1;
  const int per = (pieces + p.strips * WARPS - 1) / (p.strips * WARPS), p0 = min(pieces, (strip * WARPS + warp) * per),
            p1 = min(pieces, p0 + per);
  const uint4* wide = reinterpret_cast<const uint4*>(x - skew);
  uint8_t* ring = strip_ring + warp * STAGES * STAGE;
  // 16 bytes that lie in the row whole: pieces of memory first .. last - 1
  const int first = skew ? 1 : 0, last = (int)(((int64_t)vocab + skew) / VEC);
  const int inside_fetch = min(last, p1 + 1) - 32 * P - 1, inside = min(p1, whole) - 32 * P;         // rounds up to these need no look at ends
  const uint4* lane_wide = wide + lane;
  const uint32_t lane_ring = smem_u32(ring) + lane * 16;
  auto copy = [](uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); };
  auto fetch = [&](int c0, int stage) {              // pieces of memory c0 .. c0 + 32 P
    const uint32_t to = lane_ring + stage * STAGE;
    if (c0 >= first && c0 <= inside_fetch) {
#pragma unroll
      for (int h = 0; h < P; ++h) copy(to + h * 512, lane_wide + c0 + h * 32);
      if (skew && lane == 0) copy(to + P * 512, lane_wide + c0 + P * 32);
    } else if (c0 < p1) {
#pragma unroll 1
      for (int h = 0; h <= P; ++h) {
        const int i = h * 32 + lane, at = c0 + i;
        if (i <= 32 * P && at >= first && at < last && at <= p1) copy(to + h * 512, lane_wide + c0 + h * 32);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  float m = -kBeamFar, r = ceilf(-kBeamFar * kLog2e), s = 0.f;
  WarpList list = {0, 0};
  float least = -FLT_MAX;                            // what candidates are not below
  int held = 0;                                      // of them in list_s
  const int deep = (best + WARPS - 1) / WARPS - 1;
  volatile unsigned* bounds = bound_s;
  uint32_t tau = 0;                                  // of the list's last, once it is full
  auto tell = [&] {                                  // what this warp's list bounds
    tau = __shfl_sync(0xffffffffu, (uint32_t)((best > 32 ? list.z : list.a) >> 32), (best - 1) & 31);
    const uint32_t place = __shfl_sync(0xffffffffu, (uint32_t)(list.a >> 32), deep);
    if (lane == 0) bounds[warp] = place;
  };
  auto bound = [&](unsigned past) {                  // past = 1: elements behind those of the list lose a tie with its last
    const uint32_t all = max(__reduce_min_sync(0xffffffffu, bounds[lane % WARPS]), tau ? tau + past : 0u);
    return all ? unordered(all) : -FLT_MAX;
  };
#pragma unroll
  for (int k = 0; k < STAGES - 1; ++k) fetch(p0 + k * 32 * P, k);
  if (p0 >= p1) __syncthreads();                     // that of the others' first round; a warp without elements bounds nothing
  int stage = 0;
  for (int c0 = p0; c0 < p1; c0 += 32 * P) {
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
    __syncwarp();                                    // what lies in the stage, and that the one before has been read
    fetch(c0 + (STAGES - 1) * 32 * P, stage == 0 ? STAGES - 1 : stage - 1);
    float v[N];
    {
      const uint8_t* from = ring + stage * STAGE;
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      const uint4* at = reinterpret_cast<const uint4*>(from) + lane;
      const bool all = c0 >= first && c0 <= inside;
#pragma unroll
      for (int h = 0; h < P; ++h) {
        Pack<T, VEC> k;
        const int piece = c0 + h * 32 + lane;
        if (all || (piece < min(p1, whole) && piece >= first)) {
          *reinterpret_cast<uint4*>(&k) = skew == 0 ? at[h * 32] : load_skewed(at + h * 32, bytes);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) k.v[e] = from_f<T>(-INFINITY);
          if (piece < p1) {                          // a row's first or last
#pragma unroll
            for (int e = 0; e < VEC; ++e)
              if ((int64_t)piece * VEC + e < vocab) k.v[e] = x[(int64_t)piece * VEC + e];
          }
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
      const float to = ceilf(high * kLog2e);
      s *= power2(r - to);
      m = high;
      r = to;
    }
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float2 y = make_float2(v[e], v[e + 1]);
      const float2 z = __ffma2_rn(y, make_float2(kLog2e, kLog2e), make_float2(-r, -r));
      sum[e >> 1 & 1] = __fadd2_rn(sum[e >> 1 & 1], make_float2(exp2_approx(z.x), exp2_approx(z.y)));
    }
    s += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
    // Candidates: above the list's last (later elements of the same value lose the tie), and not below what the block's lists
    // hold together: all warps' elements at place best / 8 and before are `best` at least.  They are held back, and
    // put in the list kStripHeld or more at a time: a bound that is somewhat old lets through a few more, which costs less than a
    // list that is always up to date (16 rows' groups of 300,000: 67.1 us with 8, 75.2 with 1, 67.7 with 16, 69.4 with 32).
    auto key = [&](int i, bool in) {
      return in ? beam_key(high, (uint32_t)((c0 + i / VEC * 32 + lane) * VEC + i % VEC)) : 0;
    };
    int e = 0;
    auto first_of_high = [&] {                       // the first element of the lane's largest value
      e = N - 1;
#pragma unroll
      for (int i = N - 2; i >= 0; --i) e = v[i] == high ? i : e;
    };
    auto without = [&] {                             // the lane's largest without it
      float next = -INFINITY;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = i == e ? -INFINITY : v[i];
        next = fmaxf(next, v[i]);
      }
      high = next;
    };
    if (c0 == p0) {
      // At first the lanes' largest elements, and a bound from all warps'.
      first_of_high();
      take_lanes(list, key(e, high > -INFINITY), best);
      tell();
      __syncthreads();
      least = bound(0);
      without();
    } else {
      if (!__any_sync(0xffffffffu, high >= least)) continue;
      least = fmaxf(least, bound(1));
    }
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool in = v[i] >= least;
      e = in ? i : e;
      n += in;
    }
    const bool single = !__any_sync(0xffffffffu, n > 1);               // mostly no lane has two
#pragma unroll 1
    for (uint32_t who; (who = __ballot_sync(0xffffffffu, high >= least)) != 0;) {
      if (!single) first_of_high();
      if (high >= least) list_s[warp][held + __popc(who & ((1u << lane) - 1))] = key(e, true);
      held += __popc(who);
      if (held >= kStripHeld) {
        __syncwarp();
        take_lanes(list, lane < held ? list_s[warp][lane] : 0, best);
        const uint64_t rest = list_s[warp][32 + lane];
        __syncwarp();
        list_s[warp][lane] = rest;
        __syncwarp();
        held = max(held - 32, 0);
        tell();
        least = fmaxf(least, bound(0));
      }
      if (single) break;
      without();
    }
  }
  __syncwarp();
  if (held > 0) take_lanes(list, lane < held ? list_s[warp][lane] : 0, best);
  __syncwarp();
  if (lane < best) list_s[warp][lane] = list.a;
  if (lane + 32 < best) list_s[warp][lane + 32] = list.z;
  // the threads' sums
  float high = r;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, d));
  if (lane == 0) high_s[warp] = high;
  __syncthreads();
  high = high_s[0];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) high = fmaxf(high, high_s[w]);
  // (a power of two below what floats hold is below what counts; an infinite r, of an infinite element, has made s NaN)
  double sum = (double)(s * power2(r - high));
  bool far = false;
  if constexpr (!std::is_same_v<T, __half>) {        // (what fp16 holds is not far)
    const unsigned most = __reduce_max_sync(0xffffffffu, (unsigned)(list_s[lane % WARPS][0] >> 32));         // 0: no element above -inf
    far = most != 0 && !(fabsf(unordered(most)) <= kBeamFar);
    if (far) {                                       // +inf: NaN, as it has to be
      high = unordered(most);
      sum = beam_far_sum<T>(p, high);
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) sum_s[warp] = sum;
  // the warps' lists: a key's place is its own and what the others have above it
  uint64_t* out = p.lists + (int64_t)blockIdx.x * best;
  int taken = 0, top_half = 1;
  while (2 * top_half <= best) top_half *= 2;
  for (int i = lane; i < best; i += 32) {
    const uint64_t k = list_s[warp][i];
    if (k == 0) break;
    // all warps' lists side by side, by halves
    int place[WARPS] = {}, rank = 0;
    for (int half = top_half; half > 0; half /= 2)
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const int at = place[w] + half;
        if (at <= best && list_s[w][at - 1] > k) place[w] = at;
      }
#pragma unroll
    for (int w = 0; w < WARPS; ++w) rank += place[w];
    if (rank < best) out[rank] = k;
    ++taken;
  }
  taken = __reduce_add_sync(0xffffffffu, taken);
  if (lane == 0) have_s[warp] = taken;
  __syncthreads();
  int taken_all = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) taken_all += have_s[w];
  for (int i = taken_all + tid; i < best; i += kStripThreads) out[i] = 0;
  if (tid == 0) {
    for (int w = 1; w < WARPS; ++w) sum += sum_s[w];
    p.sums[blockIdx.x] = {sum, high, far};
  }
}

constexpr int kJoinThreads = 512;
constexpr int kJoinFew = 512;        // candidates that are compared with each other

__host__ __device__ constexpr int join_smem(int beams, int strips, int best) { return 16 * beams * best + 16 * beams * strips; }

// A row some strip of which is far: its sum beside the largest reference, which is taken off the logits before anything is added to them:
// it may be so large that nothing added to it is seen.
__device__ __noinline__ void beam_far_join(const BeamSum* sums, int strips, float score, double& base, double& from) {
  auto ref = [](const BeamSum& part) { return part.far ? (double)part.r : (double)part.r * (1. / (double)kLog2e); };
  double top = -INFINITY, sum = 0.;
  int far = 0;
  for (int s = 0; s < strips; ++s) {
    far |= sums[s].far;
    if (sums[s].s != 0.) top = fmax(top, ref(sums[s]));              // (strips without elements have a reference too)
  }
  if (!far) return;
  for (int s = 0; s < strips; ++s)
    if (sums[s].s != 0.) sum += sums[s].s * exp(ref(sums[s]) - top);
  base = (double)score - log(sum);
  from = top;
}

// One group to a block: first the strips of every row, a row to a warp, which takes the lists' places from the first on until none
// comes before its list's last; then the rows, a candidate's place being how many of the others are before it.  Bound by its chain
// of steps: what a step needs from memory is fetched a step ahead, and only candidates that some `best` are not known to
// beat look for their place.  4.3 us for 4 rows in one strip.
__global__ void __launch_bounds__(kJoinThreads) beam_join_kernel(const __grid_constant__ BeamParams p) {
  extern __shared__ __align__(16) uint64_t join_keys[];
  __shared__ double base_s[kBeamMost], from_s[kBeamMost];        // what is added to a logit, and what is taken off before
  __shared__ int taken_s, left_s, few_s[kJoinFew], reach_s[kBeamMost];
  const int tid = threadIdx.x, best = p.best, beams = p.beams, strips = p.strips;
  const int64_t group = blockIdx.x, row0 = group * beams;
  BeamSum* sums = reinterpret_cast<BeamSum*>(join_keys);                         // [beams][strips]
  uint64_t* rows = reinterpret_cast<uint64_t*>(sums + beams * strips);           // [beams][best]
  uint64_t* values = rows + beams * best;            // the same, as they are ordered: comparing 64-bit floats takes long here
  if (tid == 0) taken_s = left_s = 0;
  if (tid < kBeamMost) reach_s[tid] = 0;
  // (what the caller gave is there: the first kernel's blocks have waited for it)
  const float score = tid < beams ? p.score[row0 + tid] : 0.f;
  const bool ended = tid < beams && p.ended && p.ended[row0 + tid];
  pdl_wait();
  int far = 0;                                       // (of rows that have ended, too: whatever was there)
  for (int i = tid; i < beams * strips; i += kJoinThreads) {
    sums[i] = p.sums[row0 * strips + i];
    far |= sums[i].far;
  }
  if (strips == 1) {
    for (int i = tid; i < beams * best; i += kJoinThreads) rows[i] = p.lists[row0 * best + i];
  } else {
    const int lane = tid & 31, log = 32 - __clz(strips - 1), strip = lane & ((1 << log) - 1), places = 32 >> log;
    for (int b = tid >> 5; b < beams; b += kJoinThreads / 32) {
      const uint64_t* from = p.lists + ((row0 + b) * strips + strip) * best;
      auto fetch = [&](int place) { return strip < strips && place < best ? from[place] : 0; };
      WarpList list = {0, 0};
      uint64_t last = 0, next = fetch(lane >> log);
      for (int i = lane >> log; __any_sync(0xffffffffu, next > last); i += places) {
        const uint64_t k = next;
        next = fetch(i + places);
        take_lanes(list, k, best);
        last = list_at(list, best - 1);
      }
      if (lane < best) rows[b * best + lane] = list.a;
      if (lane + 32 < best) rows[b * best + 32 + lane] = list.z;
    }
  }
  far = __syncthreads_or(far);
  // 64-bit arithmetic is slow here: one logarithm for all rows
  if (tid < beams) {
    if (ended) {
      for (int i = 0; i < best; ++i) rows[tid * best + i] = i == 0 ? beam_key(0.f, (uint32_t)p.end) : 0;
      base_s[tid] = (double)score;
      from_s[tid] = 0.;
    } else {
      float top = -INFINITY;
      for (int s = 0; s < strips; ++s) top = fmaxf(top, sums[tid * strips + s].r);
      double sum = 0.;
      for (int s = 0; s < strips; ++s) {
        const BeamSum part = sums[tid * strips + s];
        if (part.s != 0.) sum += part.s * (double)power2(part.r - top);
      }
      base_s[tid] = (double)score - ((double)top + log2(sum)) * (1. / (double)kLog2e);
      from_s[tid] = 0.;
      if (far) beam_far_join(sums + tid * strips, strips, score, base_s[tid], from_s[tid]);
    }
  }
  __syncthreads();
  for (int i = tid; i < beams * best; i += kJoinThreads) {
    const uint64_t k = rows[i];
    double x = (double)unordered((uint32_t)(k >> 32));
    if (far) x -= from_s[i / best];
    const double v = k ? base_s[i / best] + x : -INFINITY;
    const uint64_t u = (uint64_t)__double_as_longlong(v + 0.);
    values[i] = !(v > -INFINITY) ? 0 : u >> 63 ? ~u : u | 1ull << 63;        // 0: none, or NaN
  }
  __syncthreads();
  // What is not wanted: below the largest of the rows' first values that `best` values reach, or below the rows' least at place
  // best / beams, as those and what is before them are `best`.
  for (int i = tid; i < beams * beams; i += kJoinThreads) {
    const int b = i / beams, c = i - b * beams;
    const uint64_t v = values[b * best];
    if (v) atomicAdd(&reach_s[b], above(values + c * best, best, v - 1));
  }
  __syncthreads();
  const int deep = (best + beams - 1) / beams - 1, lane = tid & 31;
  uint64_t least = ~0ull, first = 0;
  for (int b = lane; b < beams; b += 32) {
    least = min(least, values[b * best + deep]);
    if (reach_s[b] >= best) first = max(first, values[b * best]);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    least = min(least, __shfl_xor_sync(0xffffffffu, least, d));
    first = max(first, __shfl_xor_sync(0xffffffffu, first, d));
  }
  least = max(least, first);
  for (int i = tid; i < beams * best; i += kJoinThreads)
    if (values[i] != 0 && values[i] >= least) {
      const int at = atomicAdd(&left_s, 1);
      if (at < kJoinFew) few_s[at] = i;
    }
  __syncthreads();
  const int left = left_s;
  int taken = 0;
  auto put = [&](int i, int rank) {
    const int64_t o = group * best + rank;
    const uint64_t v = values[i];
    p.out_score[o] = (float)__longlong_as_double((long long)(v >> 63 ? v & ~(1ull << 63) : ~v));
    p.out_parent[o] = i / best;
    p.out_token[o] = (int)~(uint32_t)rows[i];
    ++taken;
  };
  if (left <= kJoinFew) {                            // few: each is compared with all
    for (int x = tid; x < left; x += kJoinThreads) {
      const int i = few_s[x];
      const uint64_t v = values[i];
      int rank = 0;
#pragma unroll 4
      for (int y = 0; y < left; ++y) {
        const int j = few_s[y];
        const uint64_t u = values[j];
        rank += u > v || (u == v && j < i);
      }
      if (rank < best) put(i, rank);
    }
  } else {
    int steps = 1;
    while (1 << steps <= best) ++steps;
    for (int i = tid; i < beams * best; i += kJoinThreads) {
      const uint64_t v = values[i];
      if (v == 0 || v < least) continue;
      const int b = i / best;
      int rank = i - b * best;
      for (int c0 = 0; c0 < beams && rank < best; c0 += 4) {
        // four lists side by side: falling; of equal values those of lower rows come first
        int a[4] = {0, 0, 0, 0}, z[4] = {best, best, best, best};
        for (int s = 0; s < steps; ++s)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int c = min(c0 + x, beams - 1), mid = (a[x] + z[x]) / 2;
            const uint64_t y = values[c * best + min(mid, best - 1)];
            const bool before = a[x] < z[x] && (c < b ? y >= v : y > v);
            a[x] = before ? mid + 1 : a[x];
            z[x] = before ? z[x] : mid;
          }
#pragma unroll
        for (int x = 0; x < 4; ++x) rank += c0 + x < beams && c0 + x != b ? a[x] : 0;
      }
      if (rank < best) put(i, rank);
    }
  }
  if (taken) atomicAdd(&taken_s, taken);
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
// is read once for each different parent, however many continue it.  Bound by HBM: open pages of 52 rows of 512 slots, eight
// layers of 4 heads of 128: 56 us, 5.9 TB/s (87 % of a copy's rate); 512 rows of 32 KB into another buffer: 7.2 us, 4.7 TB/s.
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

// Columns [c0, n) in steps of `step`: place(c) is where column c lies in a slot, from[i] and to[i] where slot i lies.
template <int W, typename Place>
__device__ __forceinline__ void move_columns(int64_t c0, int64_t n, int64_t step, const int8_t* parent, uint64_t need, uint64_t get,
                                             uint8_t* mine, char* const* from, char* const* to, Place place) {
  using Word = typename MoveWord<W>::type;
  const uint32_t mine32 = smem_u32(mine);
  for (int64_t c = c0; c < n; c += step) {
    const int64_t at = place(c);
    for (uint64_t b = need; b; b &= b - 1) {
      const int i = __ffsll((long long)b) - 1;
      if constexpr (W == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine32 + i * (kMoveThreads * W)), "l"(from[i] + at) : "memory");
      else if constexpr (W == 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(mine32 + i * (kMoveThreads * W)), "l"(from[i] + at) : "memory");
      else
        mine[i * (kMoveThreads * W)] = *reinterpret_cast<const uint8_t*>(from[i] + at);
    }
    if constexpr (W > 1) asm volatile("cp.async.wait_all;" ::: "memory");
    for (uint64_t b = get; b; b &= b - 1) {
      const int i = __ffsll((long long)b) - 1;
      *reinterpret_cast<Word*>(to[i] + at) = *reinterpret_cast<const Word*>(mine + parent[i] * (kMoveThreads * W));
    }
  }
}

// Blocks: segment by segment of a group of a state or pool (the last: the table).
__global__ void __launch_bounds__(kMoveThreads) beam_move_kernel(const __grid_constant__ MoveParams p) {
  extern __shared__ __align__(16) uint8_t move_smem[];
  __shared__ int8_t parent_s[kBeamMost];
  __shared__ char *from_s[kBeamMost], *to_s[kBeamMost];          // the slots' rows, or open pages
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
  const int len = paged ? len_s : 0, full = len >> p.shift, part = len & ((1 << p.shift) - 1);
  if (paged && (uneven_s || len < 0 || full > p.table_width || (full == p.table_width && part > 0))) {
    if (tid == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);            // whether anything moves or not
    return;
  }
  if (get == 0) return;
  const int64_t c0 = (int64_t)segment * kMoveThreads + tid, step = (int64_t)p.segments * kMoveThreads;
  if (!paged) {
    const MoveState& s = p.state[what];
    if (tid < p.beams) {
      from_s[tid] = s.data + (first + tid) * s.stride;
      to_s[tid] = s.out + (first + tid) * s.out_stride;
    }
    __syncthreads();
    auto go = [&](auto w) {
      constexpr int W = decltype(w)::value;
      move_columns<W>(c0, s.bytes / W, step, parent_s, need, get, move_smem + tid * W, from_s, to_s, [](int64_t c) { return c * W; });
    };
    if (s.width == 16) go(std::integral_constant<int, 16>());
    else if (s.width == 4) go(std::integral_constant<int, 4>());
    else go(std::integral_constant<int, 1>());
    return;
  }
  if (part > 0 && tid < p.beams) {                   // the open page of each slot; nothing writes its entry
    const int e = p.table[(first + tid) * p.table_stride + full];
    if (e < 0 || e >= p.n_pages) bad_s = 1;
    if (what < p.pools) from_s[tid] = p.pool[what].data + ((int64_t)e << p.shift) * p.pool[what].row_bytes;
  }
  if (what == p.pools && tid < p.beams) from_s[tid] = reinterpret_cast<char*>(p.table + (first + tid) * p.table_stride);
  __syncthreads();
  if (bad_s) {
    if (tid == 0) atomicOr(p.err, DEV_ERR_INDEX_RANGE);
    return;
  }
  if (what == p.pools) {                             // entries of full pages
    move_columns<4>(c0, full, step, parent_s, need, get, move_smem + tid * 4, from_s, from_s, [](int64_t c) { return c * 4; });
    return;
  }
  if (part == 0) return;
  const MovePages& s = p.pool[what];
  auto go = [&](auto w) {
    constexpr int W = decltype(w)::value;
    const unsigned piece = (unsigned)p.dim_bytes / W, row = piece * (unsigned)s.heads;
    move_columns<W>(c0, (int64_t)part * row, step, parent_s, need, get, move_smem + tid * W, from_s, from_s, [&](int64_t c) {
      const unsigned r = (unsigned)c / row, in = (unsigned)c - r * row, h = in / piece;
      return r * s.row_bytes + h * s.head_bytes + (int64_t)((in - h * piece) * W);
    });
  };
  if (s.width == 16) go(std::integral_constant<int, 16>());
  else if (s.width == 4) go(std::integral_constant<int, 4>());
  else go(std::integral_constant<int, 1>());
}

}  // namespace gnn
