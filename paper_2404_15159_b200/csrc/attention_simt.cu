// Masked attention in fp32 (check mode): forward and backward on the SIMT units, 64 x 64 tiles.  Formulas and masks as
// in the tensor-core kernels; every sum is fp32 and every gradient is summed by one block in one order.  Its busiest SM
// issues in 94 % of its slots, many of them loads: a thread has 4 x 4 results, for which the products read up to five times
// from shared memory for 16 multiply-adds; and dk, dv are few and long blocks.  Measured: 700 rows in 5 sequences, 8 / 4
// heads of 64, bidirectional: forward 32 us, backward 92 us.
#include "attention.cuh"

namespace mixlora {
namespace {

constexpr int kT = 64;                           // query rows and keys of a tile
constexpr int kThreads = 256;                    // thread (ty, tx): rows 4 ty + i, columns tx + 16 c  (i, c < 4)
constexpr int kPitchP = kT + 4;
template <int DP> constexpr int kPitch = DP + 4; // rows 16 bytes apart modulo the banks: 8 rows of float4 do not collide

// 64 rows of a head into shared memory; zeros behind `valid` rows and behind head_dim
template <int DP>
__device__ __forceinline__ void load_rows(float* dst, const float* src, long long stride, int valid, int head_dim) {
  for (int i = threadIdx.x; i < kT * (DP / 4); i += kThreads) {
    const int r = i / (DP / 4), c = (i % (DP / 4)) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < valid && c < head_dim) v = *reinterpret_cast<const float4*>(src + (size_t)r * stride + c);
    *reinterpret_cast<float4*>(dst + r * kPitch<DP> + c) = v;
  }
}
// The same in two steps, so that a tile's loads travel while the one before is worked on.
template <int DP>
struct RowsAhead {
  static constexpr int kPer = kT * (DP / 4) / kThreads;
  float4 v[kPer];
  __device__ __forceinline__ void fetch(const float* src, long long stride, int valid, int head_dim) {
#pragma unroll
    for (int n = 0; n < kPer; ++n) {
      const int i = n * kThreads + threadIdx.x, r = i / (DP / 4), c = (i % (DP / 4)) * 4;
      v[n] = r < valid && c < head_dim ? *reinterpret_cast<const float4*>(src + (size_t)r * stride + c)
                                       : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ void put(float* dst) const {
#pragma unroll
    for (int n = 0; n < kPer; ++n) {
      const int i = n * kThreads + threadIdx.x, r = i / (DP / 4), c = (i % (DP / 4)) * 4;
      *reinterpret_cast<float4*>(dst + r * kPitch<DP> + c) = v[n];
    }
  }
};
// acc[i][c] = A[4 ty + i] . B[tx + 16 c]
template <int DP>
__device__ __forceinline__ void dot_tile(const float* A, const float* B, int ty, int tx, float (&acc)[4][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[i][c] = 0.f;
#pragma unroll 4
  for (int d = 0; d < DP; d += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(A + (4 * ty + i) * kPitch<DP> + d);
#pragma unroll
    for (int c = 0; c < 4; ++c) y[c] = *reinterpret_cast<const float4*>(B + (tx + 16 * c) * kPitch<DP> + d);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        acc[i][c] = fmaf(x[i].w, y[c].w, fmaf(x[i].z, y[c].z, fmaf(x[i].y, y[c].y, fmaf(x[i].x, y[c].x, acc[i][c]))));
  }
}
// acc[i][4 c + e] += sum_j P(4 ty + i, j) V[j][64 c + 4 tx + e];  P by rows (ROWS) or by columns
template <int DP, bool ROWS>
__device__ __forceinline__ void sum_tile(const float* P, const float* V, int ty, int tx, float (&acc)[4][DP / 16]) {
#pragma unroll 4
  for (int j = 0; j < kT; ++j) {
    float p[4];
    if (ROWS) {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = P[(4 * ty + i) * kPitchP + j];
    } else {
      const float4 q = *reinterpret_cast<const float4*>(P + j * kPitchP + 4 * ty);
      p[0] = q.x; p[1] = q.y; p[2] = q.z; p[3] = q.w;
    }
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
      const float4 v = *reinterpret_cast<const float4*>(V + j * kPitch<DP> + c * 64 + 4 * tx);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[i][4 * c] = fmaf(p[i], v.x, acc[i][4 * c]);
        acc[i][4 * c + 1] = fmaf(p[i], v.y, acc[i][4 * c + 1]);
        acc[i][4 * c + 2] = fmaf(p[i], v.z, acc[i][4 * c + 2]);
        acc[i][4 * c + 3] = fmaf(p[i], v.w, acc[i][4 * c + 3]);
      }
    }
  }
}
template <int DP>
__device__ __forceinline__ void store_rows(float* dst, long long stride, int valid, int head_dim, int ty, int tx,
                                           const float (&acc)[4][DP / 16], const float (&mul)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
      const int at = c * 64 + 4 * tx;
      if (4 * ty + i < valid && at < head_dim)
        *reinterpret_cast<float4*>(dst + (size_t)(4 * ty + i) * stride + at) =
            make_float4(acc[i][4 * c] * mul[i], acc[i][4 * c + 1] * mul[i], acc[i][4 * c + 2] * mul[i], acc[i][4 * c + 3] * mul[i]);
    }
}
// The score in base 2 of a raw product, and the slope of the cap.  In check mode the cap goes through tanhf.
__device__ __forceinline__ float score2(const AttnArgs& a, float raw, float slope2, int distance, float& cap_slope) {
  cap_slope = 1.f;
  float x = raw * a.scale;
  if (a.softcap > 0.f) {
    const float t = tanhf(x / a.softcap);
    cap_slope = 1.f - t * t;
    x = a.softcap * t;
  }
  x *= kLog2e;
  return a.slopes ? x - slope2 * fabsf((float)distance) : x;
}
__device__ __forceinline__ bool block_tile(const int32_t* off, int n_seqs, int rows, int tile, int* seq, int* index) {
  __shared__ int found[2];
  if (threadIdx.x < 32) {
    int b = -1, t = 0;
    if (!find_tile(off, n_seqs, rows, kT, tile, &b, &t)) b = -1;
    if (threadIdx.x == 0) { found[0] = b; found[1] = t; }
  }
  __syncthreads();
  *seq = found[0];
  *index = found[1];
  return *seq >= 0;
}
__device__ __forceinline__ float max16(float v) {
#pragma unroll
  for (int f = 8; f >= 1; f >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, f));
  return v;
}
__device__ __forceinline__ float sum16(float v) {
#pragma unroll
  for (int f = 8; f >= 1; f >>= 1) v += __shfl_xor_sync(0xffffffffu, v, f);
  return v;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 2) attn_fwd_simt_kernel(AttnArgs a) {
  extern __shared__ __align__(16) float smem_f[];
  float* qs = smem_f;
  float* kv = qs + kT * kPitch<DP>;              // K, then V of the tile
  float* ps = kv + kT * kPitch<DP>;
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int head = blockIdx.x % a.q_heads, kvh = head / a.group, d = a.head_dim;
  int seq, index;
  if (!block_tile(a.q_off, a.n_seqs, a.q_rows, blockIdx.x / a.q_heads, &seq, &index)) return;
  const AttnSeq sq = load_seq(a, seq);
  const int i0 = index * kT, rows = min(kT, sq.lq - i0), p0 = sq.shift + i0;
  const KeyTiles<kT> tiles = key_tiles<kT>(sq, a.causal, a.window, p0, p0 + rows - 1);
  load_rows<DP>(qs, reinterpret_cast<const float*>(a.q) + (size_t)(sq.q0 + i0) * a.q_stride + (size_t)head * d, a.q_stride, rows, d);
  const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.f;
  float o[4][DP / 16], m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) o[i][c] = 0.f;
  }
  for (int it = 0; it < tiles.count(); ++it) {
    const int j0 = tiles.at(it) * kT, valid = min(kT, sq.lk - j0);
    const size_t krow = (size_t)(sq.k0 + j0);
    load_rows<DP>(kv, reinterpret_cast<const float*>(a.k) + krow * a.k_stride + (size_t)kvh * d, a.k_stride, valid, d);
    __syncthreads();
    float s[4][4];
    dot_tile<DP>(qs, kv, ty, tx, s);
    __syncthreads();                             // K has been read
    load_rows<DP>(kv, reinterpret_cast<const float*>(a.v) + krow * a.v_stride + (size_t)kvh * d, a.v_stride, valid, d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pos = p0 + 4 * ty + i;
      const RowKeys keys = row_keys(sq, a.causal, a.window, pos);
      float mt = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = j0 + tx + 16 * c;
        float cs;
        s[i][c] = keys.sees(j) ? score2(a, s[i][c], slope2, pos - j, cs) : -INFINITY;
        mt = fmaxf(mt, s[i][c]);
      }
      mt = max16(mt);
      if (mt > m[i]) {
        const float f = m[i] == -INFINITY ? 0.f : exp2f(m[i] - mt);
        m[i] = mt;
        l[i] *= f;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) o[i][c] *= f;
      }
      const float base = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float e = exp2f(s[i][c] - base);
        l[i] += e;
        ps[(4 * ty + i) * kPitchP + tx + 16 * c] = e;
      }
    }
    __syncthreads();
    sum_tile<DP, true>(ps, kv, ty, tx, o);
    __syncthreads();
  }
  float inv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    l[i] = sum16(l[i]);
    inv[i] = l[i] > 0.f || l[i] != l[i] ? 1.f / l[i] : 0.f;
    const int r = 4 * ty + i;
    if (a.lse && tx == 0 && r < rows) a.lse[(size_t)head * a.q_rows + sq.q0 + i0 + r] = (m[i] + log2f(l[i])) * kLn2;
  }
  store_rows<DP>(reinterpret_cast<float*>(a.out) + (size_t)(sq.q0 + i0) * a.o_stride + (size_t)head * d, a.o_stride, rows, d,
                 ty, tx, o, inv);
}

// p and ds of a tile of 64 rows (at i0) and 64 keys (at j0): p into `ps` (if not NULL), ds into `dss`.
template <int DP>
__device__ __forceinline__ void grad_tile(const AttnArgs& a, const AttnSeq& sq, int head, float slope2, int i0, int j0,
                                          const float* qs, const float* dos, const float* ks, const float* vs, float* ps,
                                          float* dss, int ty, int tx) {
  float row_lse[4], row_delta[4];                // on their way during the products
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i0 + 4 * ty + i;
    const size_t at = (size_t)head * a.q_rows + sq.q0 + (r < sq.lq ? r : 0);
    row_lse[i] = r < sq.lq ? a.lse2[at] : INFINITY;
    row_delta[i] = r < sq.lq ? a.delta[at] : 0.f;
  }
  float s[4][4], dp[4][4];
  dot_tile<DP>(qs, ks, ty, tx, s);
  dot_tile<DP>(dos, vs, ty, tx, dp);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i0 + 4 * ty + i, pos = sq.shift + r;
    const bool on = r < sq.lq;
    const RowKeys keys = row_keys(sq, a.causal, a.window, pos);
    const float lse2 = row_lse[i], delta = row_delta[i];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int j = j0 + tx + 16 * c;
      float cs, p = 0.f, ds = 0.f;
      if (on && keys.sees(j)) {
        p = exp2f(score2(a, s[i][c], slope2, pos - j, cs) - lse2);
        ds = p * (dp[i][c] - delta) * cs;
      }
      if (ps) ps[(4 * ty + i) * kPitchP + tx + 16 * c] = p;
      dss[(4 * ty + i) * kPitchP + tx + 16 * c] = ds;
    }
  }
}

template <int DP>
__device__ __forceinline__ void bwd_kv_block(const AttnArgs& a, int block, float* smem_f) {
  float* ks = smem_f;
  float* vs = ks + kT * kPitch<DP>;
  float* qs = vs + kT * kPitch<DP>;
  float* dos = qs + kT * kPitch<DP>;
  float* ps = dos + kT * kPitch<DP>;
  float* dss = ps + kT * kPitchP;
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int kvh = block % a.kv_heads, d = a.head_dim;
  int seq, index;
  if (!block_tile(a.k_off, a.n_seqs, a.k_rows, block / a.kv_heads, &seq, &index)) return;
  const AttnSeq sq = load_seq(a, seq);
  const int j0 = index * kT, keys = min(kT, sq.lk - j0);
  if (keys <= 0) return;                         // behind the used part of a slot
  int lo, hi;
  query_rows(sq, a.causal, a.window, j0, j0 + keys, &lo, &hi);
  const size_t krow = (size_t)(sq.k0 + j0);
  load_rows<DP>(ks, reinterpret_cast<const float*>(a.k) + krow * a.k_stride + (size_t)kvh * d, a.k_stride, keys, d);
  load_rows<DP>(vs, reinterpret_cast<const float*>(a.v) + krow * a.v_stride + (size_t)kvh * d, a.v_stride, keys, d);
  float dk[4][DP / 16], dv[4][DP / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) dk[i][c] = dv[i][c] = 0.f;
  const int first = lo / kT * kT, per_head = hi > first ? (hi - first + kT - 1) / kT : 0, n = per_head * a.group;
  RowsAhead<DP> nq, ndo;
  auto fetch = [&](int i) {
    const int head = kvh * a.group + i / per_head, i0 = first + (i % per_head) * kT;
    const size_t row = (size_t)(sq.q0 + i0);
    nq.fetch(reinterpret_cast<const float*>(a.q) + row * a.q_stride + (size_t)head * d, a.q_stride, sq.lq - i0, d);
    ndo.fetch(reinterpret_cast<const float*>(a.d_o) + row * a.o_stride + (size_t)head * d, a.o_stride, sq.lq - i0, d);
  };
  if (n > 0) fetch(0);
  for (int i = 0; i < n; ++i) {
    const int head = kvh * a.group + i / per_head, i0 = first + (i % per_head) * kT;
    nq.put(qs);
    ndo.put(dos);
    __syncthreads();
    if (i + 1 < n) fetch(i + 1);
    grad_tile<DP>(a, sq, head, a.slopes ? a.slopes[head] * kLog2e : 0.f, i0, j0, qs, dos, ks, vs, ps, dss, ty, tx);
    __syncthreads();
    sum_tile<DP, false>(ps, dos, ty, tx, dv);
    sum_tile<DP, false>(dss, qs, ty, tx, dk);
    __syncthreads();
  }
  const float one[4] = {1.f, 1.f, 1.f, 1.f}, mul[4] = {a.scale, a.scale, a.scale, a.scale};
  store_rows<DP>(reinterpret_cast<float*>(a.dv) + krow * a.v_stride + (size_t)kvh * d, a.v_stride, keys, d, ty, tx, dv, one);
  store_rows<DP>(reinterpret_cast<float*>(a.dk) + krow * a.k_stride + (size_t)kvh * d, a.k_stride, keys, d, ty, tx, dk, mul);
}

template <int DP>
__device__ __forceinline__ void bwd_q_block(const AttnArgs& a, int block, float* smem_f) {
  float* qs = smem_f;
  float* dos = qs + kT * kPitch<DP>;
  float* ks = dos + kT * kPitch<DP>;
  float* vs = ks + kT * kPitch<DP>;
  float* dss = vs + kT * kPitch<DP>;
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const int head = block % a.q_heads, kvh = head / a.group, d = a.head_dim;
  int seq, index;
  if (!block_tile(a.q_off, a.n_seqs, a.q_rows, block / a.q_heads, &seq, &index)) return;
  const AttnSeq sq = load_seq(a, seq);
  const int i0 = index * kT, rows = min(kT, sq.lq - i0), p0 = sq.shift + i0;
  const KeyTiles<kT> tiles = key_tiles<kT>(sq, a.causal, a.window, p0, p0 + rows - 1);
  const size_t row = (size_t)(sq.q0 + i0);
  load_rows<DP>(qs, reinterpret_cast<const float*>(a.q) + row * a.q_stride + (size_t)head * d, a.q_stride, rows, d);
  load_rows<DP>(dos, reinterpret_cast<const float*>(a.d_o) + row * a.o_stride + (size_t)head * d, a.o_stride, rows, d);
  const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.f;
  float dq[4][DP / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) dq[i][c] = 0.f;
  const int n = tiles.count();
  RowsAhead<DP> nk, nv;
  auto fetch = [&](int it) {
    const int j0 = tiles.at(it) * kT, valid = min(kT, sq.lk - j0);
    const size_t krow = (size_t)(sq.k0 + j0);
    nk.fetch(reinterpret_cast<const float*>(a.k) + krow * a.k_stride + (size_t)kvh * d, a.k_stride, valid, d);
    nv.fetch(reinterpret_cast<const float*>(a.v) + krow * a.v_stride + (size_t)kvh * d, a.v_stride, valid, d);
  };
  if (n > 0) fetch(0);
  for (int it = 0; it < n; ++it) {
    nk.put(ks);
    nv.put(vs);
    __syncthreads();
    if (it + 1 < n) fetch(it + 1);
    grad_tile<DP>(a, sq, head, slope2, i0, tiles.at(it) * kT, qs, dos, ks, vs, nullptr, dss, ty, tx);
    __syncthreads();
    sum_tile<DP, true>(dss, ks, ty, tx, dq);
    __syncthreads();
  }
  const float mul[4] = {a.scale, a.scale, a.scale, a.scale};
  store_rows<DP>(reinterpret_cast<float*>(a.dq) + row * a.q_stride + (size_t)head * d, a.q_stride, rows, d, ty, tx, dq, mul);
}

// dk, dv and dq in one launch: the key blocks, which are fewer and longer, start first.
template <int DP>
__global__ void __launch_bounds__(kThreads, 1) attn_bwd_simt_kernel(AttnArgs a, int key_blocks) {
  extern __shared__ __align__(16) float smem_f[];
  if ((int)blockIdx.x < key_blocks) bwd_kv_block<DP>(a, blockIdx.x, smem_f);
  else bwd_q_block<DP>(a, blockIdx.x - key_blocks, smem_f);
}

template <int DP> constexpr int bytes(int rows, int tiles) { return 4 * (rows * kT * kPitch<DP> + tiles * kT * kPitchP); }

template <int DP>
cudaError_t forward(const AttnArgs& a, long long grid, cudaStream_t st) {
  static bool done[64];
  cudaError_t e = allow_smem(attn_fwd_simt_kernel<DP>, bytes<DP>(2, 1), done);
  if (e != cudaSuccess || grid == 0) return e;
  attn_fwd_simt_kernel<DP><<<(unsigned)grid, kThreads, bytes<DP>(2, 1), st>>>(a);
  return cudaGetLastError();
}
template <int DP>
cudaError_t backward(const AttnArgs& a, long long key_blocks, long long row_blocks, cudaStream_t st) {
  static bool done[64];
  cudaError_t e = allow_smem(attn_bwd_simt_kernel<DP>, bytes<DP>(4, 2), done);
  if (e != cudaSuccess || key_blocks + row_blocks == 0) return e;
  attn_bwd_simt_kernel<DP><<<(unsigned)(key_blocks + row_blocks), kThreads, bytes<DP>(4, 2), st>>>(a, (int)key_blocks);
  return cudaGetLastError();
}
long long tiles_of(int rows, int n_seqs, int heads) {
  return rows ? ((long long)(rows + kT - 1) / kT + n_seqs) * heads : 0;
}

}  // namespace

cudaError_t launch_attn_forward_simt(const AttnArgs& a, cudaStream_t st) {
  const long long grid = tiles_of(a.q_rows, a.n_seqs, a.q_heads);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  return a.head_dim <= 64 ? forward<64>(a, grid, st) : forward<128>(a, grid, st);
}

cudaError_t launch_attn_backward_simt(const AttnArgs& a, cudaStream_t st) {
  const long long gk = tiles_of(a.k_rows, a.n_seqs, a.kv_heads), gq = tiles_of(a.q_rows, a.n_seqs, a.q_heads);
  if (gk + gq > 0x7fffffffLL) return cudaErrorInvalidValue;
  return a.head_dim <= 64 ? backward<64>(a, gk, gq, st) : backward<128>(a, gk, gq, st);
}

}  // namespace mixlora
