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

constexpr int kThreads = 256;

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

// One item: N values at each of two places of a head (half layout: i and i + rotary_dim / 2), or N neighbouring
// values (interleaved layout, and the copied rest).  With N values of 16 bytes and both places of an item read before
// either is written, the kernel also works in place.
template <typename T, int N, bool INTERLEAVED>
struct Item {
  const T* src;
  T* dst;
  int at;              // first value of the item inside its head
  int cs;              // index of its first pair in the cos / sin table, or -1: copied
  bool on;
  Vec<T, N> a, b;

  __device__ __forceinline__ void load(int half) {
    if (!on) return;
    a = *reinterpret_cast<const Vec<T, N>*>(src + at);
    if (!INTERLEAVED && cs >= 0) b = *reinterpret_cast<const Vec<T, N>*>(src + at + half);
  }
  __device__ __forceinline__ void store(int half, const float2* table) {
    if (!on) return;
    if (cs >= 0) {
      if (INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const float2 t = table[cs + e / 2];
          const float u = to_f(a.v[e]), w = to_f(a.v[e + 1]);
          a.v[e] = from_f<T>(u * t.x - w * t.y);
          a.v[e + 1] = from_f<T>(w * t.x + u * t.y);
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 t = table[cs + e];
          const float u = to_f(a.v[e]), w = to_f(b.v[e]);
          a.v[e] = from_f<T>(u * t.x - w * t.y);
          b.v[e] = from_f<T>(w * t.x + u * t.y);
        }
        *reinterpret_cast<Vec<T, N>*>(dst + at + half) = b;
      }
    }
    *reinterpret_cast<Vec<T, N>*>(dst + at) = a;
  }
};

// Bound by memory: every value is read and written once.  A block takes `block_tokens` tokens (and, where there are
// few tokens, a share of the heads, gridDim.y): its threads first make the tokens' cos and sin once for all heads, in
// shared memory, then walk over (token, head, item) with kUnroll items' loads in flight each.
// The angle's turns are formed and reduced in 64 bits; the rest of a turn goes through sincospif in 32.
template <typename T, int N, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs p) {
  extern __shared__ float2 cs_table[];                  // [block_tokens, pairs]
  constexpr int kUnroll = 4;
  const int t0 = blockIdx.x * p.block_tokens;
  const int nt = min(p.block_tokens, p.tokens - t0);
  const int heads = p.q_heads + p.k_heads;
  const int h0 = (int)((long long)heads * blockIdx.y / gridDim.y);
  const int h1 = (int)((long long)heads * (blockIdx.y + 1) / gridDim.y);
  const int half = p.pairs;
  const int rot_items = INTERLEAVED ? 2 * p.pairs / N : p.pairs / N;
  const int items = rot_items + p.copied / N;           // per head
  const int per_token = items * (h1 - h0);
  const int total = per_token * nt;

  Item<T, N, INTERLEAVED> it[kUnroll];
  int table_row[kUnroll];
  auto fetch = [&](int first) {
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int idx = first + j * kThreads;
      it[j].on = idx < total;
      if (!it[j].on) continue;
      const int tl = idx / per_token, rest = idx - tl * per_token;
      const int hl = rest / items, i = rest - hl * items;
      const int h = h0 + hl;
      const size_t row = (size_t)(t0 + tl);
      if (h < p.q_heads) {
        it[j].src = reinterpret_cast<const T*>(p.q) + row * p.q_stride + (size_t)h * p.head_dim;
        it[j].dst = reinterpret_cast<T*>(p.q_out) + row * p.q_out_stride + (size_t)h * p.head_dim;
      } else {
        it[j].src = reinterpret_cast<const T*>(p.k) + row * p.k_stride + (size_t)(h - p.q_heads) * p.head_dim;
        it[j].dst = reinterpret_cast<T*>(p.k_out) + row * p.k_out_stride + (size_t)(h - p.q_heads) * p.head_dim;
      }
      if (i < rot_items) {
        it[j].at = i * N;
        it[j].cs = INTERLEAVED ? i * (N / 2) : i * N;
      } else {
        it[j].at = 2 * p.pairs + (i - rot_items) * N;
        it[j].cs = -1;
      }
      table_row[j] = tl * p.pairs;
      it[j].load(half);
    }
  };
  fetch(threadIdx.x);                                   // the first items travel while the table is made
  for (int i = threadIdx.x; i < nt * p.pairs; i += kThreads) {
    const int tl = i / p.pairs, pr = i - tl * p.pairs;
    const double pos = p.positions ? (double)p.positions[t0 + tl] : (double)(t0 + tl);
    const double turns = pos * (p.inv_freq[pr] * 0.15915494309189535);
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs_table[i] = make_float2(c * p.amplitude, s * (p.backward ? -p.amplitude : p.amplitude));
  }
  __syncthreads();
  for (int first = threadIdx.x; first < total; first += kThreads * kUnroll) {
    if (first != (int)threadIdx.x) fetch(first);
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) it[j].store(half, cs_table + (it[j].on ? table_row[j] : 0));
  }
}

template <typename T, int N, bool IL>
cudaError_t launch(const RopeArgs& p, dim3 grid, size_t smem, cudaStream_t st) {
  rope_kernel<T, N, IL><<<grid, kThreads, smem, st>>>(p);
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
  // Tokens per block: 4 share one round of the table's work; with fewer than four blocks per SM the tokens go one by
  // one, and with few tokens the heads are spread over up to 8 blocks so that a decoding step uses more SMs.
  const int sms = 148;
  p.block_tokens = p.tokens >= 16 * sms ? 4 : 1;
  const int blocks = (p.tokens + p.block_tokens - 1) / p.block_tokens;
  int split = 1;
  while (split < 8 && (long long)blocks * split < sms && p.q_heads + p.k_heads >= 8 * split) split *= 2;
  const dim3 grid((unsigned)blocks, (unsigned)split);
  const size_t smem = (size_t)p.block_tokens * p.pairs * sizeof(float2);
  if (bf16_mode) {
    if (wide) return interleaved ? launch<bf16, 8, true>(p, grid, smem, st) : launch<bf16, 8, false>(p, grid, smem, st);
    return interleaved ? launch<bf16, 2, true>(p, grid, smem, st) : launch<bf16, 1, false>(p, grid, smem, st);
  }
  if (wide) return interleaved ? launch<float, 4, true>(p, grid, smem, st) : launch<float, 4, false>(p, grid, smem, st);
  return interleaved ? launch<float, 2, true>(p, grid, smem, st) : launch<float, 1, false>(p, grid, smem, st);
}

}  // namespace mixlora
