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
// factor in two floats, each exact as an FMA pair.  16-bit results take the hardware's sine and cosine of that
// angle (absolute error below 2^-21 within half a turn, theirs is 2^-9 or 2^-12), fp32 results sincospif.
//
// Bound by HBM: every element is read and written once.  A group of lanes owns a row of units for two heads of a
// token, so that a thread has up to 64 bytes on their way, and little else: an angle's sine and cosine are used
// for both heads and forgotten, and computed again for the token's next two.  Keeping them through all heads took
// 118 registers and left 15 warps to an SM.  Queries, keys and values are different blocks' work; frequencies and
// gains lie in shared memory.  300,000 rows of two bf16 heads of 64: 27 us, 84 % of the copy rate (43 us with the
// angles kept); with norms, keys and values 74 us, 92 % (137 us).  In fp32 51 us, 89 %, and 144 us, 94 %.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <type_traits>
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
  unsigned block0[4];                // the parts' first blocks, and all blocks
  int dim, rot, units, group;        // units of a row, lanes that share it (a power of two)
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
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
  T v[N];
  __device__ __forceinline__ float2 get2(int i) const { return make_float2(to_f(v[i]), to_f(v[i + 1])); }
  __device__ __forceinline__ void set2(int i, float2 x) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      *reinterpret_cast<__nv_bfloat162*>(v + i) = __floats2bfloat162_rn(x.x, x.y);
    } else if constexpr (std::is_same<T, __half>::value) {
      *reinterpret_cast<__half2*>(v + i) = __floats2half2_rn(x.x, x.y);
    } else {
      v[i] = x.x;
      v[i + 1] = x.y;
    }
  }
};

// x (hi + lo) turns, less whole turns.
__device__ __forceinline__ float turns_real(float x, float hi, float lo) {
  const float a = x * hi, ea = fmaf(x, hi, -a), b = x * lo, eb = fmaf(x, lo, -b);
  return (a - rintf(a)) + ((ea - rintf(ea)) + (b - rintf(b)) + eb);
}
__device__ __forceinline__ float turns_whole(int x, uint64_t fixed) {
  return (float)(int)((fixed * (uint64_t)(int64_t)x + 0x80000000u) >> 32) * 0x1p-32f;
}

// V pairs to a unit.  V == 1 takes any even R and any alignment that elements have; larger V need R and D to
// be multiples of 2V and addresses and strides of V elements.
template <typename T, int V, bool INTER, bool NORM>
__global__ void __launch_bounds__(kRotThreads, V >= 8 ? 4 : 5) rotary_kernel(const __grid_constant__ RotaryParams p) {
  constexpr int UPL = V >= 4 ? 1 : 4 / V;          // units a lane may own: D <= 256
  constexpr int MOST = 2 * kRotMaxPairs / (2 * V); // units of a row
  __shared__ uint64_t freq_s[V][MOST];             // fixed, or hi and lo as the two halves
  __shared__ float gain_s[NORM ? 2 * V : 1][MOST];
  const int part = blockIdx.x < p.block0[1] ? 0 : blockIdx.x < p.block0[2] ? 1 : 2;
  const unsigned block = blockIdx.x - p.block0[part], blocks = p.block0[part + 1] - p.block0[part];
  const int heads = p.heads[part];
  const unsigned twos = (unsigned)(heads + 1) / 2;
  const bool copy = part == 2;
  const int sub = threadIdx.x & (p.group - 1), pairs = p.rot / 2;
  for (int i = threadIdx.x; i < pairs; i += kRotThreads)
    freq_s[i % V][i / V] = p.pos_float ? (uint64_t)__float_as_uint(p.hi[i]) << 32 | __float_as_uint(p.lo[i]) : p.fixed[i];
  pdl_wait();
  if (NORM && !copy) {
    const float* gain = p.gain[part];
    for (int i = threadIdx.x; i < p.units; i += kRotThreads) {
      const bool half = !INTER && i * V < pairs;
#pragma unroll 1
      for (int e = 0; e < V; ++e) {
        gain_s[e][i] = gain ? gain[(half ? i * V : 2 * i * V) + e] : 1.f;
        gain_s[V + e][i] = gain ? gain[(half ? i * V + pairs : 2 * i * V + V) + e] : 1.f;
      }
    }
  }
  __syncthreads();
  const int64_t groups = (int64_t)blocks * (kRotThreads / p.group), tasks = p.tokens * twos;
  const int64_t first = (int64_t)block * (kRotThreads / p.group) + threadIdx.x / p.group;
  for (int64_t task = first; __any_sync(0xffffffffu, task < tasks); task += groups) {   // the same rounds for a whole warp
    const int64_t at = min(task, tasks - 1);
    const int64_t t = twos == 1 ? at : tasks >> 32 ? at / twos : (int64_t)((uint32_t)at / twos);
    const int h = 2 * (int)(at - t * twos);
    const bool both = h + 1 < heads;
    const char* x = p.in[part].data + t * p.in[part].row_bytes + (int64_t)h * p.in[part].head_bytes;
    Pack<T, V> xu[2][UPL], xw[2][UPL];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int u = 0; u < UPL; ++u) {
        const int unit = sub + u * p.group, i = unit * V;
        const bool half = !INTER && i < pairs;
        if (unit < p.units && (b == 0 || both)) {
          const char* head = x + b * p.in[part].head_bytes;
          xu[b][u] = *reinterpret_cast<const Pack<T, V>*>(head + (half ? i : 2 * i) * sizeof(T));
          xw[b][u] = *reinterpret_cast<const Pack<T, V>*>(head + (half ? i + pairs : 2 * i + V) * sizeof(T));
        }
      }
    const int64_t row = part == 0 || !p.rows ? t : p.rows[t];
    const bool store = task < tasks && (part == 0 || !p.rows || (row >= 0 && row < p.out_rows));
    if (!copy) {
      const int pos = !p.pos ? (int)t : static_cast<const int*>(p.pos)[t];     // or a float's bits
      float r[2] = {1.f, 1.f};
      if (NORM) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float2 sum = make_float2(0.f, 0.f);
#pragma unroll
          for (int u = 0; u < UPL; ++u)
            if (sub + u * p.group < p.units) {
              if constexpr (V == 1) {
                const float2 v = make_float2(to_f(xu[b][u].v[0]), to_f(xw[b][u].v[0]));
                sum = __ffma2_rn(v, v, sum);
              } else {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                  const float2 v = xu[b][u].get2(e), w = xw[b][u].get2(e);
                  sum = __ffma2_rn(v, v, sum);
                  sum = __ffma2_rn(w, w, sum);
                }
              }
            }
          r[b] = sum.x + sum.y;
        }
        for (int m = p.group >> 1; m > 0; m >>= 1) {
          r[0] += __shfl_xor_sync(0xffffffffu, r[0], m);
          r[1] += __shfl_xor_sync(0xffffffffu, r[1], m);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) r[b] = rsqrtf(r[b] / (float)p.dim + p.eps);
      }
#pragma unroll
      for (int u = 0; u < UPL; ++u) {
        const int unit = sub + u * p.group;
        if (unit >= p.units) continue;
        if (unit * V >= pairs) {                   // past the rotation: each element by itself, whatever lies beside it
          if constexpr (NORM) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int e = 0; e < V; ++e) {
                xu[b][u].v[e] = from_f<T>(to_f(xu[b][u].v[e]) * (r[b] * gain_s[e][unit]));
                xw[b][u].v[e] = from_f<T>(to_f(xw[b][u].v[e]) * (r[b] * gain_s[V + e][unit]));
              }
          }
          continue;
        }
        auto angle = [&](int e, float& c, float& s) {
          const uint64_t f = freq_s[e][unit];
          const float turns = p.pos_float ? turns_real(__int_as_float(pos), __uint_as_float((uint32_t)(f >> 32)),
                                                       __uint_as_float((uint32_t)f))
                                          : turns_whole(pos, f);
          if (sizeof(T) == 4) {
            sincospif(2.f * turns, &s, &c);
          } else {
            const float a = 6.2831853071795865f * (turns - rintf(turns));
            s = __sinf(a);
            c = __cosf(a);
          }
          c *= p.amplitude;
          s *= p.amplitude;
        };
        if constexpr (V == 1) {
          float c, s;
          angle(0, c, s);
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            float a = to_f(xu[b][u].v[0]), d = to_f(xw[b][u].v[0]);
            if (NORM) {
              a *= r[b] * gain_s[0][unit];
              d *= r[b] * gain_s[1][unit];
            }
            xu[b][u].v[0] = from_f<T>(a * c - d * s);
            xw[b][u].v[0] = from_f<T>(d * c + a * s);
          }
        } else {
#pragma unroll
          for (int e = 0; e < V; e += 2) {         // pairs e and e + 1
            float2 c, s;
            angle(e, c.x, s.x);
            angle(e + 1, c.y, s.y);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              if constexpr (INTER) {               // elements 2e .. 2e + 3, which lie in u, then in w
                Pack<T, V>& at_e = 2 * e < V ? xu[b][u] : xw[b][u];
                const int i = 2 * e % V;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  if constexpr (V == 2) {
                    Pack<T, V>& y = k ? xw[b][u] : xu[b][u];
                    float2 z = y.get2(0);
                    if (NORM) z = make_float2(z.x * (r[b] * gain_s[2 * k][unit]), z.y * (r[b] * gain_s[2 * k + 1][unit]));
                    const float cc = k ? c.y : c.x, ss = k ? s.y : s.x;
                    y.set2(0, make_float2(z.x * cc - z.y * ss, z.y * cc + z.x * ss));
                  } else {
                    float2 z = at_e.get2(i + 2 * k);
                    if (NORM)
                      z = make_float2(z.x * (r[b] * gain_s[2 * (e + k)][unit]), z.y * (r[b] * gain_s[2 * (e + k) + 1][unit]));
                    const float cc = k ? c.y : c.x, ss = k ? s.y : s.x;
                    at_e.set2(i + 2 * k, make_float2(z.x * cc - z.y * ss, z.y * cc + z.x * ss));
                  }
                }
              } else {
                float2 a = xu[b][u].get2(e), d = xw[b][u].get2(e);
                if (NORM) {
                  const float2 rr = make_float2(r[b], r[b]);
                  a = __fmul2_rn(a, __fmul2_rn(rr, make_float2(gain_s[e][unit], gain_s[e + 1][unit])));
                  d = __fmul2_rn(d, __fmul2_rn(rr, make_float2(gain_s[V + e][unit], gain_s[V + e + 1][unit])));
                }
                const float2 ds = __fmul2_rn(d, s), as = __fmul2_rn(a, s);
                xu[b][u].set2(e, __ffma2_rn(a, c, make_float2(-ds.x, -ds.y)));
                xw[b][u].set2(e, __ffma2_rn(d, c, as));
              }
            }
          }
        }
      }
    }
    if (!store) continue;
    char* y = p.out[part].data + row * p.out[part].row_bytes + (int64_t)h * p.out[part].head_bytes;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int u = 0; u < UPL; ++u) {
        const int unit = sub + u * p.group, i = unit * V;
        const bool half = !INTER && i < pairs;
        if (unit < p.units && (b == 0 || both)) {
          char* head = y + b * p.out[part].head_bytes;
          *reinterpret_cast<Pack<T, V>*>(head + (half ? i : 2 * i) * sizeof(T)) = xu[b][u];
          *reinterpret_cast<Pack<T, V>*>(head + (half ? i + pairs : 2 * i + V) * sizeof(T)) = xw[b][u];
        }
      }
  }
}

}  // namespace gnn
