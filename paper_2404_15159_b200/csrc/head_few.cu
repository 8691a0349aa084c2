// The two products for a few tokens (up to 64; bf16): bound by reading the head, once each.
//
// The roles of the operands are turned around: 128 columns of the vocabulary are the rows of a tensor-core tile, the tokens
// its columns (16, 32 or 64), so that no part of a tile is empty and the head streams through shared memory at the rate of
// the memory.  One persistent CTA an SM; warp 0 loads (128 reduction elements a stage, so that 256 bytes of each row are
// asked for at once), warp 1 issues the products, warps 2 to 5 add up the stages' sums in registers, rounded to nearest (the
// tensor core, which cuts off what is behind 24 bits, runs up to 8 stages ahead of them), and pass the tile through shared
// memory, and warps 2 to 9 then work on a token each, four neighbouring columns a lane.
// Rows are tokens here: those that are left out pass through the products too, and the joining kernel drops them.
//
// The gradient's product goes the same way: 256 columns of d_x are the rows of two tiles, the tokens their columns, and the
// vocabulary, which is the reduction, is shared out so that every SM has one item.  The shares' sums go to memory, and a
// kernel of their own adds them up in their order (a few MB that L2 holds; one CTA a tile would read them for 10 us).
// Measured on a B200, 32000 columns, width 4096 (262 MB): logits of one token 48 us (5.5 TB/s, the copy rate is 6.56), of 64
// tokens with their exponentials 55; the gradient of 16 tokens 44 us and 6 for its sums.  What is left is the first loads'
// latency and the last tile's results; 250 tiles on 148 SMs cost nothing, since those that are left share the memory.
#include <cuda.h>
#include <math.h>

#include "head.cuh"
#include "tc_ptx.cuh"

namespace mixlora {
namespace {

using namespace tc;
constexpr int kWarps = 8, kThreads = 64 + 32 * kWarps, kBK = 64, kUmmaK = 16;
// A stage is a span of 128 products, and of the stages that take turns in an accumulator every second one goes on in it with its
// products subtracted (see the kernel for many tokens).  In registers four stages are added up to one another before the tile's
// sum, whose own roundings are kept for up to 16 tokens (with 32 that took 55.6 -> 57.2 us).  On logits whose products lean by
// 0.3 of their spread, width 4096: too small by 0.15 units of 2^-23 with a spread of 0.3 (up to 16 tokens) and 0.5, where spans
// of 512 that do not turn gave 4.4, and fp32's own products 0 and 1.1.
constexpr int kBufs = 8;                                  // accumulators, one a stage
__device__ __forceinline__ bool goes_back(int stage) { return (stage / kBufs) & 1; }
constexpr uint32_t kABytes = 2 * 128 * kBK * 2;
template <int NC> struct Few {
  static constexpr uint32_t kBBytes = 2 * NC * kBK * 2, kStage = kABytes + kBBytes;
  static constexpr int kStages = NC == 16 ? 6 : (NC == 32 ? 5 : 4);
  static constexpr uint32_t kTurn = NC * kHeadCols * 4;   // the finished tile, [token][column]
  static constexpr uint32_t kSmem = kStages * kStage + kTurn + 1024 + 256;
};
struct alignas(64) FewMaps { CUtensorMap w, x; };

template <int NC, bool GRAD, bool CAP>
__global__ void __launch_bounds__(kThreads, 1) head_few_kernel(const __grid_constant__ HeadArgs p,
                                                               const __grid_constant__ FewMaps maps) {
  using F = Few<NC>;
  constexpr int kStages = F::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* turn = reinterpret_cast<float*>(smem + kStages * F::kStage);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * F::kStage + F::kTurn);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kStages + 2 * kBufs);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* give_up = abort_flag + 1;                 // one of the result warps waited in vain
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem), bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto tfull_bar = [&](int b) { return bar_base + 8u * (kStages + b); };
  auto tempty_bar = [&](int b) { return bar_base + 8u * (kStages + kBufs + b); };

  let_next_start();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(full_bar(s), 1);
    for (int b = 0; b < kBufs; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 4); }
    *abort_flag = 0;
    *give_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tmap(&maps.w); prefetch_tmap(&maps.x);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), kBufs * NC);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.state->status = 0;
    p.state->joined = 0;
  }

  const int steps = (p.d + 2 * kBK - 1) / (2 * kBK);
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < p.col_tiles && ok; tile += gridDim.x) {
        for (int s = 0; s < steps; ++s, ++it) {
          const int st = it % kStages;
          // a stage is free when the products that read it have arrived, `kStages` before these
          if (it >= kStages && !mbar_wait(tfull_bar((it - kStages) % kBufs), ((it - kStages) / kBufs) & 1u, abort_flag)) {
            ok = false;
            break;
          }
          const uint32_t a_dst = smem_base + st * F::kStage, b_dst = a_dst + kABytes;
          mbar_expect_tx(full_bar(st), F::kStage);
          const int k = s * 2 * kBK;
          tma_load_2d(a_dst, &maps.w, full_bar(st), k, tile * kHeadCols);
          tma_load_2d(a_dst + kABytes / 2, &maps.w, full_bar(st), k + kBK, tile * kHeadCols);
          tma_load_2d(b_dst, &maps.x, full_bar(st), k, 0);
          tma_load_2d(b_dst + F::kBBytes / 2, &maps.x, full_bar(st), k + kBK, 0);
        }
      }
      if (!ok) {
        *abort_flag = 1;
        atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = make_idesc(NC, 0, 0);
      constexpr uint32_t kNegateA = 1u << 13;
      uint32_t it = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < p.col_tiles && ok; tile += gridDim.x) {
        for (int s = 0; s < steps; ++s, ++it) {
          const int st = it % kStages, buf = it % kBufs;
          if (!mbar_wait(tempty_bar(buf), ((it / kBufs) & 1u) ^ 1u, abort_flag) ||
              !mbar_wait(full_bar(st), (it / kStages) & 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t acc = tmem_base + buf * NC;
          const bool back = goes_back(s);
          const uint32_t a_addr = smem_base + st * F::kStage, b_addr = a_addr + kABytes;
#pragma unroll
          for (int k = 0; k < 2 * kBK / kUmmaK; ++k) {
            const uint32_t half = k / (kBK / kUmmaK), in = k % (kBK / kUmmaK);
            umma_bf16(acc, make_desc(a_addr + half * (kABytes / 2) + in * (kUmmaK * 2), 16, 1024),
                      make_desc(b_addr + half * (F::kBBytes / 2) + in * (kUmmaK * 2), 16, 1024),
                      back ? idesc | kNegateA : idesc, back || k > 0);
          }
          umma_commit(tfull_bar(buf));
        }
      }
      if (!ok) {
        *abort_flag = 1;
        atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
      }
    }
  } else {
    wait_for_last();                                      // for the lists: the products need the call's inputs alone
    constexpr int kLow = NC == 16 ? NC : 1;
    const int q = warp & 3;
    const float factor = p.logit_factor, cap_out = p.cap_out, to2 = p.to2;
    uint32_t count = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < p.col_tiles && ok; tile += gridDim.x) {
      float x[NC], some[NC];                              // the tile's sums, and those of the last four stages
      float low[kLow];                                    // what the roundings of the tile's sums have left, up to 16 tokens
      if (warp < 6) {
#pragma unroll
        for (int j = 0; j < NC; ++j) x[j] = some[j] = low[j % kLow] = 0.f;
        for (int s = 0; s < steps; ++s, ++count) {
          const uint32_t buf = count % kBufs, use = count / kBufs;
          if (!__all_sync(0xffffffffu, mbar_wait(tfull_bar(buf), use & 1u, abort_flag))) { ok = false; break; }
          tc_fence_after();
          const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + buf * NC;
          const float times = goes_back(s) ? -1.f : (s + kBufs < steps ? 2.f : 1.f);
#pragma unroll
          for (int c = 0; c < NC; c += 16) {
            uint32_t v[16];
            tmem_ld16(acc + c, v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) some[c + j] = fmaf(__uint_as_float(v[j]), times, some[c + j]);
          }
          if (s % 4 == 3 || s == steps - 1) {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
              const float sum = x[j] + some[j], of_some = sum - x[j];
              if (kLow == NC) low[j % kLow] += (x[j] - (sum - of_some)) + (some[j] - of_some);
              x[j] = sum;
              some[j] = 0.f;
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(tempty_bar(buf));
        }
      }
      // the warps meet whether a wait ran out or not, and leave together
      if (!ok) *give_up = 1;
      named_barrier(1, 32 * kWarps);                      // the tile before has been read
      ok = *give_up == 0;
      if (warp < 6) {
#pragma unroll
        for (int j = 0; j < NC; ++j) turn[j * kHeadCols + q * 32 + lane] = kLow == NC ? x[j] + low[j % kLow] : x[j];
      }
      named_barrier(1, 32 * kWarps);
      if (!ok) break;
      const int n0 = tile * kHeadCols, col = n0 + lane * 4;
      for (int t = warp - 2; t < min(NC, p.tokens); t += kWarps) {
        const float4 f = *reinterpret_cast<const float4*>(turn + t * kHeadCols + lane * 4);
        float v[4] = {f.x, f.y, f.z, f.w};
        uint32_t dead = 0;                                // of this lane's columns: listed, or behind the vocabulary
#pragma unroll
        for (int j = 0; j < 4; ++j) dead |= col + j >= p.vocab ? 1u << j : 0u;
        const int32_t* list = p.list + (size_t)t * p.top;
        for (int k0 = 0; k0 < p.top; k0 += 32) {
          const int c = k0 + lane < p.top ? list[k0 + lane] : kHeadNone;
          unsigned hit = __ballot_sync(0xffffffffu, c >= n0 && c < n0 + kHeadCols && c < p.vocab);
          while (hit) {
            const int l = __ffs(hit) - 1, at = __shfl_sync(0xffffffffu, c, l) - n0;
            hit &= hit - 1;
            if (at >> 2 == lane) {
              const int j = at & 3;
              const float raw = (j == 0 ? v[0] : j == 1 ? v[1] : j == 2 ? v[2] : v[3]) * factor;
              p.z_listed[(size_t)t * p.top + k0 + l] = fmaf(raw, 0.f, CAP ? tanhf(raw) * cap_out : raw);
              dead |= 1u << j;
            }
          }
        }
        float most = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!(dead >> j & 1)) most = fmaxf(most, v[j]);
#pragma unroll
        for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        most *= factor;
        if (CAP) most = tanhf(most) * cap_out;
        const float r = most == -INFINITY ? 0.f : kHeadStep * rintf(most * (1.4426950408889634f / kHeadStep));
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float ex, slope = 1.f;
          if (CAP) {
            const float th = tanhf(v[j] * factor);
            ex = exp2_fast(fmaf(th, to2, -r));
            slope = (1.f - th) * (1.f + th);
          } else {
            ex = exp2_fast(fmaf(v[j], to2, -r));
          }
          sum += dead >> j & 1 ? 0.f : fmaf(v[j], 0.f, ex);      // no number where the product is infinite
          if (dead >> j & 1) ex = 0.f;
          v[j] = CAP ? ex * slope : ex;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) p.stats[(size_t)t * p.col_tiles + tile] = make_float2(r, sum);
        if (GRAD && col < p.pitch) {
          const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), up = __floats2bfloat162_rn(v[2], v[3]);
          *reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(p.e) + (size_t)t * p.pitch + col) =
              make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&up));
        }
      }
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
    }
  }

  __syncthreads();
  if (*abort_flag) {
    for (int i = 0; i < 200; ++i) __nanosleep(5000);      // let copies that may still be in flight land
  }
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem_base, kBufs * NC);
  }
}

// ---- the gradient's product ----
constexpr int kOut = 256;                                 // columns of d_x of an item
template <int NC> struct FewGrad {
  static constexpr uint32_t kABytes = kOut * kBK * 2, kBBytes = NC * kBK * 2, kStage = kABytes + kBBytes;
  static constexpr int kStages = NC == 64 ? 5 : 6;
  static constexpr uint32_t kSmem = kStages * kStage + 1024 + 256;
  static constexpr uint32_t kTmem = 2 * NC < 32 ? 32 : 2 * NC;
};

template <int NC>
__global__ void __launch_bounds__(192, 1) head_few_grad_kernel(const __grid_constant__ HeadArgs p,
                                                               const __grid_constant__ FewMaps maps, int shares) {
  using F = FewGrad<NC>;
  constexpr int kStages = F::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * F::kStage);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem), bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (kStages + s); };
  const uint32_t done_bar = bar_base + 8u * (2 * kStages);

  let_next_start();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(done_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tmap(&maps.w); prefetch_tmap(&maps.x);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), F::kTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  const int tile = blockIdx.x / shares, share = blockIdx.x - tile * shares, c0 = tile * kOut;
  const int blocks = (p.vocab + kBK - 1) / kBK;
  const int kb0 = (int)((long long)share * blocks / shares), kb1 = (int)((long long)(share + 1) * blocks / shares);
  if (warp == 0) {
    if (lane == 0) {
      auto load_w = [&](int kb, int st) {
        mbar_expect_tx(full_bar(st), F::kStage);
        for (int j = 0; j < kOut / 64; ++j)
          tma_load_2d(smem_base + st * F::kStage + j * (kBK * 128), &maps.w, full_bar(st), c0 + 64 * j, kb * kBK);
      };
      auto load_e = [&](int kb, int st) {
        tma_load_2d(smem_base + st * F::kStage + F::kABytes, &maps.x, full_bar(st), kb * kBK, 0);
      };
      // the head is nobody's result: its first blocks come in while the rows are still being joined
      const int early = min(kStages, kb1 - kb0);
      for (int i = 0; i < early; ++i) load_w(kb0 + i, i);
      wait_for_last();
      for (int i = 0; i < early; ++i) load_e(kb0 + i, i);
      bool ok = true;
      for (int kb = kb0 + early, it = early; kb < kb1; ++kb, ++it) {
        const int st = it % kStages;
        if (!mbar_wait(empty_bar(st), ((it / kStages) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        load_w(kb, st);
        load_e(kb, st);
      }
      if (!ok) {
        *abort_flag = 1;
        atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      wait_for_last();
      const uint32_t idesc = make_idesc(NC, 1, 0);
      bool ok = true;
      for (int kb = kb0, it = 0; kb < kb1; ++kb, ++it) {
        const int st = it % kStages;
        if (!mbar_wait(full_bar(st), (it / kStages) & 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t a_addr = smem_base + st * F::kStage, b_addr = a_addr + F::kABytes;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int k = 0; k < kBK / kUmmaK; ++k)
            umma_bf16(tmem_base + sub * NC, make_desc(a_addr + sub * (2 * kBK * 128) + k * (kUmmaK * 128), kBK * 128, 1024),
                      make_desc(b_addr + k * (kUmmaK * 2), 16, 1024), idesc, kb > kb0 || k > 0);
        umma_commit(empty_bar(st));
      }
      if (ok) {
        umma_commit(done_bar);
      } else {
        *abort_flag = 1;
        atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
      }
    }
  } else {
    wait_for_last();
    const int q = warp & 3;
    if (__all_sync(0xffffffffu, mbar_wait(done_bar, 0, abort_flag))) {
      tc_fence_after();
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const int c = c0 + sub * 128 + q * 32 + lane;
        float* to = p.part + (size_t)share * p.tokens * p.d + c;
#pragma unroll
        for (int t = 0; t < NC; t += 16) {
          uint32_t v[16];
          tmem_ld16(tmem_base + ((uint32_t)(q * 32) << 16) + sub * NC + t, v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (c < p.d && t + j < p.tokens) to[(size_t)(t + j) * p.d] = __uint_as_float(v[j]);
        }
      }
      tc_fence_before();
    } else if (lane == 0) {
      *abort_flag = 1;
      atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
    }
  }
  __syncthreads();
  if (*abort_flag) {
    for (int i = 0; i < 200; ++i) __nanosleep(5000);      // let copies that may still be in flight land
  }
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem_base, F::kTmem);
  }
}

// d_x from the shares, eight columns of a token a thread
__global__ void __launch_bounds__(128) head_few_add_kernel(HeadArgs p, int shares) {
  let_next_start();
  wait_for_last();
  const int each = p.d / 8;
  const int i = blockIdx.x * 128 + threadIdx.x;
  if (i >= p.tokens * each) return;
  const int t = i / each, c = (i - t * each) * 8;
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (p.token_row[t] >= 0) {
    const float* from = p.part + (size_t)t * p.d + c;
    const size_t apart = (size_t)p.tokens * p.d;
#pragma unroll 8
    for (int s = 0; s < shares; ++s) {
      const float4 a = __ldcg(reinterpret_cast<const float4*>(from + s * apart));
      const float4 b = __ldcg(reinterpret_cast<const float4*>(from + s * apart + 4));
      sum[0] += a.x; sum[1] += a.y; sum[2] += a.z; sum[3] += a.w;
      sum[4] += b.x; sum[5] += b.y; sum[6] += b.z; sum[7] += b.w;
    }
    const float by = p.row_scale[t];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] *= by;
  }
  uint4 out;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&out);
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(sum[2 * j], sum[2 * j + 1]);
  *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(p.d_x) + (size_t)t * p.dx_stride + c) = out;
}

template <int NC>
cudaError_t launch_grad(const HeadArgs& p, cudaStream_t st) {
  FewMaps m;
  if (!tc_encode_2d(&m.w, p.w, p.vocab, p.d, p.w_stride, kBK, 64) || !tc_encode_2d(&m.x, p.e, p.piece, p.vocab, p.pitch, NC, kBK))
    return cudaErrorInvalidValue;
  static bool done[64] = {false};
  cudaError_t e = allow_smem(head_few_grad_kernel<NC>, FewGrad<NC>::kSmem, done);
  if (e != cudaSuccess) return e;
  const int shares = head_few_shares(p.d, p.vocab), tiles = (p.d + kOut - 1) / kOut;
  e = launch_behind(head_few_grad_kernel<NC>, (unsigned)(tiles * shares), 192, FewGrad<NC>::kSmem, st, p, m, shares);
  if (e != cudaSuccess) return e;
  const int threads = p.tokens * (p.d / 8);
  return launch_behind(head_few_add_kernel, (unsigned)((threads + 127) / 128), 128, 0, st, p, shares);
}

template <int NC, bool GRAD, bool CAP>
cudaError_t launch(const HeadArgs& p, bool first, cudaStream_t st) {
  FewMaps m;
  if (!tc_encode_2d(&m.w, p.w, p.vocab, p.d, p.w_stride, kHeadCols, kBK) ||
      !tc_encode_2d(&m.x, p.x, p.tokens, p.d, p.x_stride, NC, kBK))
    return cudaErrorInvalidValue;
  static bool done[64] = {false};
  cudaError_t e = allow_smem(head_few_kernel<NC, GRAD, CAP>, Few<NC>::kSmem, done);
  if (e != cudaSuccess) return e;
  const int sms = 2 * head_pairs(), grid = p.col_tiles < sms ? p.col_tiles : sms;
  if (!first) return launch_behind(head_few_kernel<NC, GRAD, CAP>, (unsigned)grid, kThreads, Few<NC>::kSmem, st, p, m);
  head_few_kernel<NC, GRAD, CAP><<<grid, kThreads, Few<NC>::kSmem, st>>>(p, m);
  return cudaGetLastError();
}
template <int NC>
cudaError_t launch_for(const HeadArgs& p, bool first, cudaStream_t st) {
  if (p.softcap > 0.f) return p.d_x ? launch<NC, true, true>(p, first, st) : launch<NC, false, true>(p, first, st);
  return p.d_x ? launch<NC, true, false>(p, first, st) : launch<NC, false, false>(p, first, st);
}

}  // namespace

cudaError_t launch_head_logits_few(const HeadArgs& p, bool first, cudaStream_t st) {
  if (p.tokens <= 16) return launch_for<16>(p, first, st);
  if (p.tokens <= 32) return launch_for<32>(p, first, st);
  return launch_for<64>(p, first, st);
}

int head_few_shares(int d, int vocab) {
  const int tiles = (d + kOut - 1) / kOut, blocks = (vocab + kBK - 1) / kBK;
  int shares = 2 * kHeadPairs / tiles;
  if (shares > blocks / 4) shares = blocks / 4;           // no share of less than 4 blocks
  return shares > 0 ? shares : 1;
}

cudaError_t launch_head_grad_few(const HeadArgs& p, cudaStream_t st) {
  if (p.tokens <= 16) return launch_grad<16>(p, st);
  if (p.tokens <= 32) return launch_grad<32>(p, st);
  return launch_grad<64>(p, st);
}

}  // namespace mixlora
