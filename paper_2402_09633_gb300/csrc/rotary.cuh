// Rotary positions, and norms of queries and keys with the rotation in the same pass.
//
// A head of D elements is cut into units: a rotated unit is V pairs (u, w), which lie at i and i + R/2
// (half layout) or side by side (interleaved); an element past R passes unrotated, 2V to a unit.  With
// x' = x / sqrt(mean(x^2) + eps) * gain first (norm), (u, w) becomes
//   (u cos a - w sin a, w cos a + u sin a),  a = position * frequency.
// The arithmetic is fp32 and the result is rounded once.
//
// The angle is kept in turns, whole turns dropped before anything is rounded: for a whole position as the 64-bit
// product of the position and f / 2 pi in 2^-64 turns, which wraps at a turn by itself, so that no int32 position
// costs accuracy (a plain fp32 angle is off by up to 0.06 rad at 10^6); for a real one as products with the
// factor in two floats, each exact as an FMA pair.
//
// Bound by HBM: every element is read and written once.  A group of lanes owns a row of units and keeps its
// cosines and sines while it goes through the heads of a token.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "ptx.cuh"

namespace gnn {

constexpr int kRotMaxPairs = 128;
constexpr int kRotThreads = 256;

struct HeadsView {                   // [rows, heads, D], elements of a head contiguous
  char* data;
  int64_t row_bytes, head_bytes;
};

struct RotaryParams {
  HeadsView in[3], out[3];           // queries, keys (rotated, normed), values (copied)
  int heads[3];
  int dim, rot, units, group;        // units of a row, lanes that share it (a power of two)
  int chunk, chunks;                 // heads a group goes through, and how many such parts a token has
  int64_t tokens, out_rows;
  const void* pos;
  const int64_t* rows;               // where keys and values go, or null: row t
  int pos_float;
  float eps, amplitude;
  const float* gain[2];              // of queries and of keys, or null
  uint64_t fixed[kRotMaxPairs];      // turns a position, in 2^-64 turns (modulo a turn)
  float hi[kRotMaxPairs], lo[kRotMaxPairs];   // the same as a sum of floats
};

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f<__half>(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

// N contiguous elements in accesses of up to 16 bytes; the address is aligned to that.
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack { T v[N]; };

// x (hi + lo) turns, less whole turns.
__device__ __forceinline__ float turns_real(float x, float hi, float lo) {
  const float a = x * hi, ea = fmaf(x, hi, -a), b = x * lo, eb = fmaf(x, lo, -b);
  return (a - rintf(a)) + ((ea - rintf(ea)) + (b - rintf(b)) + eb);
}
__device__ __forceinline__ float turns_whole(int x, uint64_t fixed) {
  return (float)(int)((fixed * (uint64_t)(int64_t)x + 0x80000000u) >> 32) * 0x1p-32f;
}

// V pairs to a unit.  V == 1 takes any even R and any alignment that elements have; larger V need R and D to
// be multiples of 2V and addresses and strides of V elements (2V interleaved).
template <typename T, int V, bool INTER, bool NORM>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
  constexpr int UPL = V == 1 ? 4 : 1;              // units a lane may own: D <= 256
  constexpr int BATCH = V == 1 ? 1 : 2;            // heads whose loads are in flight together
  pdl_wait();
  const int sub = threadIdx.x & (p.group - 1);
  const int64_t groups = (int64_t)gridDim.x * (kRotThreads / p.group);
  const int pairs = p.rot / 2;
  int eu[UPL], ew[UPL];                            // first elements of the unit's two halves
  bool mine[UPL], turned[UPL];
  uint64_t freq[UPL][V];                           // fixed, or hi and lo as the two halves
#pragma unroll
  for (int u = 0; u < UPL; ++u) {
    const int unit = sub + u * p.group, i = unit * V;
    mine[u] = unit < p.units;
    turned[u] = mine[u] && i < pairs;
    eu[u] = turned[u] && !INTER ? i : 2 * i;
    ew[u] = turned[u] && !INTER ? i + pairs : 2 * i + V;
    if (!mine[u]) eu[u] = ew[u] = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      freq[u][e] = !turned[u] ? 0
                   : p.pos_float ? (uint64_t)__float_as_uint(p.hi[i + e]) << 32 | __float_as_uint(p.lo[i + e])
                                 : p.fixed[i + e];
    }
  }
  const int64_t tasks = p.tokens * p.chunks;
  const int64_t first = (int64_t)blockIdx.x * (kRotThreads / p.group) + threadIdx.x / p.group;
  const int64_t warp_first = first - (threadIdx.x & 31) / p.group;   // the loop is uniform in a warp
  const int n_heads = p.heads[0] + p.heads[1] + p.heads[2];
  for (int64_t w = warp_first; w < tasks; w += groups) {
    int64_t task = w + (first - warp_first);
    const bool live = task < tasks;
    if (!live) task = tasks - 1;
    const int64_t t = p.chunks == 1 ? task : task / p.chunks;
    const int h0 = p.chunks == 1 ? 0 : (int)(task - t * p.chunks) * p.chunk;
    const int h1 = min(h0 + p.chunk, n_heads);
    float c[UPL][V], s[UPL][V];
    const int whole = p.pos_float ? 0 : p.pos ? static_cast<const int*>(p.pos)[t] : (int)t;
    const float real = p.pos_float ? static_cast<const float*>(p.pos)[t] : 0.f;
#pragma unroll
    for (int u = 0; u < UPL; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint64_t f = freq[u][e];
        const float turns = p.pos_float ? turns_real(real, __uint_as_float((uint32_t)(f >> 32)), __uint_as_float((uint32_t)f))
                                        : turns_whole(whole, f);
        sincospif(2.f * turns, &s[u][e], &c[u][e]);
        c[u][e] *= p.amplitude;
        s[u][e] *= p.amplitude;
      }
    const int64_t kv_row = p.rows ? p.rows[t] : t;
    const bool kv_live = live && (!p.rows || (kv_row >= 0 && kv_row < p.out_rows));
    for (int hb = h0; hb < h0 + p.chunk; hb += BATCH) {
      Pack<T, V> xu[BATCH][UPL], xw[BATCH][UPL];
      int part[BATCH], head[BATCH];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        int h = min(hb + b, h1 - 1);
        part[b] = h < p.heads[0] ? 0 : h < p.heads[0] + p.heads[1] ? 1 : 2;
        head[b] = h - (part[b] > 0 ? p.heads[0] : 0) - (part[b] > 1 ? p.heads[1] : 0);
        const char* x = p.in[part[b]].data + t * p.in[part[b]].row_bytes + head[b] * p.in[part[b]].head_bytes;
#pragma unroll
        for (int u = 0; u < UPL; ++u)
          if (mine[u]) {
            xu[b][u] = *reinterpret_cast<const Pack<T, V>*>(x + eu[u] * sizeof(T));
            xw[b][u] = *reinterpret_cast<const Pack<T, V>*>(x + ew[u] * sizeof(T));
          }
      }
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        float r = 1.f;
        if (NORM) {
          float sum = 0.f;
#pragma unroll
          for (int u = 0; u < UPL; ++u)
            if (mine[u]) {
#pragma unroll
              for (int e = 0; e < V; ++e) {
                const float a = to_f(xu[b][u].v[e]), d = to_f(xw[b][u].v[e]);
                sum = fmaf(a, a, sum);
                sum = fmaf(d, d, sum);
              }
            }
          for (int m = p.group >> 1; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
          r = rsqrtf(sum / (float)p.dim + p.eps);
        }
        const float* gain = NORM && part[b] < 2 ? p.gain[part[b]] : nullptr;
        const bool store = hb + b < h1 && (part[b] == 0 ? live : kv_live);
        const int64_t row = part[b] == 0 ? t : kv_row;
        char* y = p.out[part[b]].data + row * p.out[part[b]].row_bytes + head[b] * p.out[part[b]].head_bytes;
#pragma unroll
        for (int u = 0; u < UPL; ++u)
          if (mine[u] && store) {
            Pack<T, V> yu = xu[b][u], yw = xw[b][u];
            if (part[b] < 2) {
              float v[2 * V];                      // elements as they lie: eu.., ew..
#pragma unroll
              for (int e = 0; e < V; ++e) {
                v[e] = to_f(yu.v[e]);
                v[V + e] = to_f(yw.v[e]);
                if (NORM) {
                  v[e] *= r;
                  v[V + e] *= r;
                  if (gain) {
                    v[e] *= gain[eu[u] + e];
                    v[V + e] *= gain[ew[u] + e];
                  }
                }
              }
#pragma unroll
              for (int e = 0; e < V; ++e) {
                float& a = v[INTER ? 2 * e : e];
                float& d = v[INTER ? 2 * e + 1 : V + e];
                const float na = a * c[u][e] - d * s[u][e], nd = d * c[u][e] + a * s[u][e];
                if (turned[u]) { a = na; d = nd; }
              }
#pragma unroll
              for (int e = 0; e < V; ++e) {
                yu.v[e] = from_f<T>(v[e]);
                yw.v[e] = from_f<T>(v[V + e]);
              }
            }
            *reinterpret_cast<Pack<T, V>*>(y + eu[u] * sizeof(T)) = yu;
            *reinterpret_cast<Pack<T, V>*>(y + ew[u] * sizeof(T)) = yw;
          }
      }
    }
  }
}

}  // namespace gnn
