// The two products of the head's losses in the fp32 check mode, on the fp32 pipes.
//
//   logits   x [rows, d] . w [vocab, d]^T, as they are, to the piece's array; the joining kernel turns them into factors
//   grad     those factors [rows, vocab] . w [vocab, d], times the row's scale, to the row's token
//
// 128 x 128 tiles, 8 x 8 results a thread as pairs along the columns (one instruction multiplies and adds two), operands
// transposed into shared memory 16 deep, the next 16 loaded into registers under this one's products.  Where the second
// product has fewer tiles than the GPU holds blocks, several blocks share a tile's reduction; the block that comes last
// adds the shares up in their order.
#include "head.cuh"

namespace mixlora {
namespace {

constexpr int kTile = 128, kDeep = 16, kThreads = 256, kPitch = kTile + 4;

typedef unsigned long long pair32;      // two fp32
__device__ __forceinline__ pair32 pack2(float a, float b) {
  pair32 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(pair32 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ pair32 fma2(pair32 a, pair32 b, pair32 c) {
  pair32 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

template <bool TO_X>
__global__ void __launch_bounds__(kThreads, 2) head_simt_kernel(HeadArgs p, int n_tiles, int shares) {
  let_next_start();
  wait_for_last();
  __shared__ __align__(16) float as[2][kDeep][kPitch], bs[2][kDeep][kPitch];
  __shared__ int last;
  const int rows = head_rows_here(p);
  const int item = blockIdx.x, share = item % shares, tile = item / shares;
  const int m0 = tile / n_tiles * kTile, n0 = (tile % n_tiles) * kTile;
  if (m0 >= rows) return;
  const int tid = threadIdx.x;
  const int depth = TO_X ? p.vocab : p.d;
  const int steps = (depth + kDeep - 1) / kDeep;
  const int s0 = (int)((long long)share * steps / shares), s1 = (int)((long long)(share + 1) * steps / shares);

  // this thread's pieces of a step: four values along k of two rows of A and, for the logits, of two rows of w
  const int lr = tid >> 2, lk = (tid & 3) * 4;
  const float *ap[2], *bp[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = m0 + lr + 64 * i;
    ap[i] = nullptr;
    if (r < rows)
      ap[i] = TO_X ? reinterpret_cast<const float*>(p.e) + (size_t)r * p.pitch
                   : reinterpret_cast<const float*>(p.x) + (size_t)p.row_token[p.piece0 + r] * p.x_stride;
    const int c = n0 + lr + 64 * i;
    bp[i] = !TO_X && c < p.vocab ? reinterpret_cast<const float*>(p.w) + (size_t)c * p.w_stride : nullptr;
  }
  float4 ra[2], rb[2];
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  auto load = [&](int step) {
    const int k = step * kDeep + lk;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ra[i] = zero;
      if (ap[i] && k < depth) {
        ra[i] = *reinterpret_cast<const float4*>(ap[i] + k);
        if (TO_X) {                                    // what lies behind the last column may be anything
          if (k + 1 >= depth) ra[i].y = 0.f;
          if (k + 2 >= depth) ra[i].z = 0.f;
          if (k + 3 >= depth) ra[i].w = 0.f;
        }
      }
      rb[i] = zero;
      if (!TO_X) {
        if (bp[i] && k < depth) rb[i] = *reinterpret_cast<const float4*>(bp[i] + k);
      } else {
        const int kr = step * kDeep + (tid >> 5) + 8 * i, c = n0 + (tid & 31) * 4;
        if (kr < depth && c < p.d)
          rb[i] = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.w) + (size_t)kr * p.w_stride + c);
      }
    }
  };
  auto keep = [&](int buf) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = lr + 64 * i;
      as[buf][lk][r] = ra[i].x; as[buf][lk + 1][r] = ra[i].y; as[buf][lk + 2][r] = ra[i].z; as[buf][lk + 3][r] = ra[i].w;
      if (!TO_X) {
        bs[buf][lk][r] = rb[i].x; bs[buf][lk + 1][r] = rb[i].y; bs[buf][lk + 2][r] = rb[i].z; bs[buf][lk + 3][r] = rb[i].w;
      } else {
        *reinterpret_cast<float4*>(&bs[buf][(tid >> 5) + 8 * i][(tid & 31) * 4]) = rb[i];
      }
    }
  };

  const int tx = tid & 15, ty = tid >> 4;              // rows ty * 4 and 64 + ty * 4, columns tx * 4 and 64 + tx * 4
  pair32 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0ull;
  if (s0 < s1) {
    load(s0);
    keep(0);
  }
  __syncthreads();
  for (int s = s0; s < s1; ++s) {
    const int buf = (s - s0) & 1;
    if (s + 1 < s1) load(s + 1);
#pragma unroll
    for (int k = 0; k < kDeep; ++k) {
      const float4 a0 = *reinterpret_cast<const float4*>(&as[buf][k][ty * 4]);
      const float4 a1 = *reinterpret_cast<const float4*>(&as[buf][k][64 + ty * 4]);
      const ulonglong2 b0 = *reinterpret_cast<const ulonglong2*>(&bs[buf][k][tx * 4]);
      const ulonglong2 b1 = *reinterpret_cast<const ulonglong2*>(&bs[buf][k][64 + tx * 4]);
      const float a[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
      const pair32 b[4] = {b0.x, b0.y, b1.x, b1.y};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const pair32 aa = pack2(a[i], a[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fma2(aa, b[j], acc[i][j]);
      }
    }
    if (s + 1 < s1) keep(buf ^ 1);
    __syncthreads();
  }

  if (TO_X && shares > 1) {
    float4* mine = reinterpret_cast<float4*>(p.part) + (size_t)item * (kTile * kTile / 4) + tid;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float4 v;
        unpack2(acc[i][2 * h], v.x, v.y);
        unpack2(acc[i][2 * h + 1], v.z, v.w);
        mine[(i * 2 + h) * kThreads] = v;
      }
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(p.counters + tile, 1) == shares - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const float4* first = reinterpret_cast<const float4*>(p.part) + (size_t)tile * shares * (kTile * kTile / 4) + tid;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float4 sum = zero;
        for (int s = 0; s < shares; ++s) {
          const float4 v = __ldcg(first + (size_t)s * (kTile * kTile / 4) + (i * 2 + h) * kThreads);
          sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
        }
        acc[i][2 * h] = pack2(sum.x, sum.y);
        acc[i][2 * h + 1] = pack2(sum.z, sum.w);
      }
    if (tid == 0) p.counters[tile] = 0;                // ready for the next piece
  }

  const int width = TO_X ? p.d : p.vocab;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = m0 + (i < 4 ? ty * 4 + i : 60 + ty * 4 + i);
    if (r >= rows) continue;
    float* out = TO_X ? reinterpret_cast<float*>(p.d_x) + (size_t)p.row_token[p.piece0 + r] * p.dx_stride
                      : reinterpret_cast<float*>(p.e) + (size_t)r * p.pitch;
    const float by = TO_X ? p.row_scale[r] : 1.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = n0 + 64 * h + tx * 4;
      float4 v;
      unpack2(acc[i][2 * h], v.x, v.y);
      unpack2(acc[i][2 * h + 1], v.z, v.w);
      v.x *= by; v.y *= by; v.z *= by; v.w *= by;
      if (c + 3 < width) {
        *reinterpret_cast<float4*>(out + c) = v;
      } else {
        if (c < width) out[c] = v.x;
        if (c + 1 < width) out[c + 1] = v.y;
        if (c + 2 < width) out[c + 2] = v.z;
      }
    }
  }
}

}  // namespace

// Both grids are sized for a piece in which every row counts; blocks without rows end at once.
cudaError_t launch_head_logits_simt(const HeadArgs& p, cudaStream_t st) {
  const int n_tiles = (p.vocab + kTile - 1) / kTile;
  const long long blocks = (long long)((p.piece + kTile - 1) / kTile) * n_tiles;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  return launch_behind(head_simt_kernel<false>, (unsigned)blocks, kThreads, 0, st, p, n_tiles, 1);
}

cudaError_t launch_head_grad_simt(const HeadArgs& p, cudaStream_t st) {
  const int n_tiles = (p.d + kTile - 1) / kTile;
  const long long tiles = (long long)((p.piece + kTile - 1) / kTile) * n_tiles;
  // two blocks an SM are what registers allow; a share keeps 8 steps of the reduction at least
  const int hold = 4 * head_pairs() < kHeadSimtShares ? 4 * head_pairs() : kHeadSimtShares, steps = (p.vocab + kDeep - 1) / kDeep;
  int shares = 1;
  while (shares < kHeadMaxShares && tiles * (shares + 1) <= hold && (shares + 1) * 8 <= steps) ++shares;
  if (tiles * shares > 0x7fffffffLL) return cudaErrorInvalidValue;
  return launch_behind(head_simt_kernel<true>, (unsigned)(tiles * shares), kThreads, 0, st, p, n_tiles, shares);
}

}  // namespace mixlora
