// Rotary positions of the attention projections: forward, the gradient's way back, and the frequencies' table.
//
// A head's leading rotary_dim values are taken as rotary_dim / 2 pairs (u, w), and pair i of a token at position p is
// turned by the angle p * w_i:  u' = u cos - w sin,  w' = w cos + u sin  (both times `amplitude`); the gradient is
// turned back by the same angle.  Values behind rotary_dim are copied.
#include <cuda_bf16.h>

#include "common.cuh"
#include "rope.cuh"

namespace mixlora {
namespace {

constexpr int kThreads = 128;

// Radians per position of every pair.  In 64 bits: positions reach millions of radians, where a frequency rounded to
// 32 bits would be off by a large part of a turn.
__global__ void rope_frequencies_kernel(int pairs, double theta, int scaling, double factor, double low, double high,
                                        double original, double* out) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= pairs) return;
  const double r = 2.0 * pairs;
  if (scaling == MIXLORA_ROPE_SCALE_NTK) theta *= pow(factor, r / (r > 2.0 ? r - 2.0 : 1.0));
  double w = pow(theta, -2.0 * i / r);
  if (scaling == MIXLORA_ROPE_SCALE_LINEAR) w /= factor;
  if (scaling == MIXLORA_ROPE_SCALE_PARTS) {
    const double turns = original * w / 6.283185307179586;
    const double keep = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
    w = w * keep + w / factor * (1.0 - keep);
  }
  out[i] = w;
}

template <typename T, int N> struct alignas(N * sizeof(T)) Vec { T v[N]; };
__device__ __forceinline__ float to_f(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(float x) { return x; }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ bf16 from_f<bf16>(float x) { return __float2bfloat16(x); }
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }

// pos * freq / (2 pi) without its whole turns.  The product and its division keep what they round off: at 2^31 radians a
// double's half step is 2^-22 already.
__device__ __forceinline__ double rest_of_turns(double pos, double freq) {
  constexpr double kPerTurn = 0.15915494309189535, kPerTurnLow = -9.839338337591243e-18;      // 1 / (2 pi) in two parts
  const double angle = pos * freq, angle_low = fma(pos, freq, -angle);
  const double turns = angle * kPerTurn;
  const double low = fma(angle, kPerTurn, -turns) + fma(angle, kPerTurnLow, angle_low * kPerTurn);
  return (turns - rint(turns)) + low;
}

// Bound by memory: every value is read and written once.  A warp takes a token (where there are few, a share of its
// heads).  Every lane keeps to one item of a head: N values at each of two places, i and i + rotary_dim / 2 (half
// layout), or N neighbouring values (interleaved, and the copied rest); it makes its pairs' cos and sin once, in
// registers, and walks over the heads with kUnroll items' loads in flight.  An item is 16 bytes where the pairs allow
// it; both places of an item are read before either is written, so the kernel also works in place.
// The angle's turns are formed and reduced in 64 bits; the rest of a turn goes through sincospif in 32: a rounding of at
// most 2^-25 half turns (pi 2^-25) and sincospif's own 2^-24 leave the sines within 2^-22.
// Measured on B200: q and k of 8192 tokens, 32 + 32 heads of 128 in bf16, 50 us (5.4 TB/s); 32768 tokens, 32 + 8 heads out
// of packed rows, 114 us (5.9 TB/s).
template <typename T, int N, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads, 8) rope_kernel(RopeArgs p) {
  // items in flight per lane: fewer registers, so more warps, beat more loads per warp in bf16 (8192 tokens: 50 us with
  // one, 53 with two, 64 with three); with half as many pairs to a lane fp32 has room for two (1021 tokens, which L2 holds: 11 and 13 us; 19 out of memory)
  constexpr int kUnroll = sizeof(T) == 2 ? 1 : 2;
  constexpr int kPairs = INTERLEAVED ? (N + 1) / 2 : N;
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int t = (int)(unit / p.shares), share = (int)(unit - (long long)t * p.shares);
  if (t >= p.tokens) return;
  const int heads = p.q_heads + p.k_heads;
  const int h0 = (int)((long long)heads * share / p.shares), h1 = (int)((long long)heads * (share + 1) / p.shares);
  const int rot_items = INTERLEAVED ? 2 * p.pairs / N : p.pairs / N;
  const int items = rot_items + p.copied / N;           // per head
  const double pos = p.positions ? (double)p.positions[t] : (double)t;
  const T* q = reinterpret_cast<const T*>(p.q) + (size_t)t * p.q_stride;
  const T* k = reinterpret_cast<const T*>(p.k) + (size_t)t * p.k_stride;
  T* q_out = reinterpret_cast<T*>(p.q_out) + (size_t)t * p.q_out_stride;
  T* k_out = reinterpret_cast<T*>(p.k_out) + (size_t)t * p.k_out_stride;

  for (int i0 = 0; i0 < items; i0 += 32) {
    const int here = min(32, items - i0), step = 32 / here;          // lanes of a head, heads of a warp
    const int hl = lane / here, i = i0 + lane - hl * here;
    if (hl >= step) continue;
    const bool turn = i < rot_items;
    const int at = turn ? i * N : 2 * p.pairs + (i - rot_items) * N;
    Vec<T, N> a[kUnroll], b[kUnroll];
    auto load = [&](int h) {
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        const int hh = h + j * step;
        if (hh >= h1) continue;
        const T* src = (hh < p.q_heads ? q + (size_t)hh * p.head_dim : k + (size_t)(hh - p.q_heads) * p.head_dim) + at;
        a[j] = *reinterpret_cast<const Vec<T, N>*>(src);
        if (!INTERLEAVED && turn) b[j] = *reinterpret_cast<const Vec<T, N>*>(src + p.pairs);
      }
    };
    float c[kPairs], s[kPairs];
    if (turn) {
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        const double turns = rest_of_turns(pos, p.inv_freq[i * kPairs + e]);
        sincospif((float)(2.0 * turns), &s[e], &c[e]);
        c[e] *= p.amplitude;
        s[e] *= p.backward ? -p.amplitude : p.amplitude;
      }
    }
    for (int h = h0 + hl; h < h1; h += step * kUnroll) {
      load(h);
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) {
        const int hh = h + j * step;
        if (hh >= h1) continue;
        T* dst = (hh < p.q_heads ? q_out + (size_t)hh * p.head_dim : k_out + (size_t)(hh - p.q_heads) * p.head_dim) + at;
        if (turn) {
          if (INTERLEAVED) {
#pragma unroll
            for (int e = 0; e + 1 < N; e += 2) {
              const float u = to_f(a[j].v[e]), w = to_f(a[j].v[e + 1]);
              a[j].v[e] = from_f<T>(u * c[e / 2] - w * s[e / 2]);
              a[j].v[e + 1] = from_f<T>(w * c[e / 2] + u * s[e / 2]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
              const float u = to_f(a[j].v[e]), w = to_f(b[j].v[e]);
              a[j].v[e] = from_f<T>(u * c[e] - w * s[e]);
              b[j].v[e] = from_f<T>(w * c[e] + u * s[e]);
            }
            *reinterpret_cast<Vec<T, N>*>(dst + p.pairs) = b[j];
          }
        }
        *reinterpret_cast<Vec<T, N>*>(dst) = a[j];
      }
    }
  }
}

template <typename T, int N, bool IL>
cudaError_t launch(const RopeArgs& p, cudaStream_t st) {
  const long long blocks = ((long long)p.tokens * p.shares + kThreads / 32 - 1) / (kThreads / 32);
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  rope_kernel<T, N, IL><<<(unsigned)blocks, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope_frequencies(int pairs, double theta, int scaling, double factor, double low, double high,
                                    double original, double* out, cudaStream_t st) {
  rope_frequencies_kernel<<<(pairs + 127) / 128, 128, 0, st>>>(pairs, theta, scaling, factor, low, high, original, out);
  return cudaGetLastError();
}

cudaError_t launch_rope(RopeArgs p, bool bf16_mode, bool interleaved, cudaStream_t st) {
  // 16 bytes per item where the pairs fall on 16-byte pieces of a head, else one pair (two values) per item
  const int n = bf16_mode ? 8 : 4;
  const bool wide = (interleaved ? 2 * p.pairs : p.pairs) % n == 0 && p.copied % n == 0;
  // With fewer tokens than the SMs hold warps of this kernel (148 x 16 of them keep the memory busy) the heads of a
  // token are spread over several warps, down to 8 heads each.
  const int heads = p.q_heads + p.k_heads;
  p.shares = 1;
  while ((long long)p.tokens * p.shares < 148 * 16 && heads >= 16 * p.shares) p.shares *= 2;
  if (bf16_mode) {
    if (wide) return interleaved ? launch<bf16, 8, true>(p, st) : launch<bf16, 8, false>(p, st);
    return interleaved ? launch<bf16, 2, true>(p, st) : launch<bf16, 1, false>(p, st);
  }
  if (wide) return interleaved ? launch<float, 4, true>(p, st) : launch<float, 4, false>(p, st);
  return interleaved ? launch<float, 2, true>(p, st) : launch<float, 1, false>(p, st);
}

}  // namespace mixlora
