// The two products of the head's losses on the tensor cores (tcgen05, TMEM, TMA; bf16 operands, fp32 accumulation).
//
//   logits   x [rows, d] . w [vocab, d]^T   per tile of 256 columns: R, S, the listed logits and, for a gradient, E
//   grad     E [rows, vocab] . w [vocab, d]  times the row's A scale / temperature weight / normalizer, to the row's token
//
// Pairs of CTAs work on 256 x 256 tiles (cta_group::2, 128 rows of the accumulator and half of B's columns each), one
// persistent pair on two SMs; warp 0 loads, warp 1 of the leader issues the products, the other warps turn a finished
// accumulator into its result while the second one is filled.  The number of rows is read on the device: tokens without a
// label take no part.
#include <cuda.h>
#include <math.h>

#include "head.cuh"
#include "tc_ptx.cuh"

namespace mixlora {
namespace {

using namespace tc;
constexpr int kBK = 64, kUmmaK = 16, kTile = kHeadTile;
constexpr int kStages = 6;
// warps that take finished accumulators: the logits need two for each quarter of the rows, 128 columns a thread
constexpr int result_warps(bool to_x) { return to_x ? 4 : 8; }
constexpr int threads_of(bool to_x) { return 64 + 32 * result_warps(to_x); }
// k-blocks of a logit that the tensor core adds up before the sum is taken on in registers (see logits_rows)
constexpr int kSpan = 16;
constexpr uint32_t kABytes = 128 * kBK * 2, kBBytes = 128 * kBK * 2, kStageBytes = kABytes + kBBytes;
constexpr uint32_t kSmemBytes = kStages * kStageBytes + 1024 + 256;
constexpr uint32_t kTmemCols = 512;
// a share of a split reduction keeps at least this many k-blocks, and costs this many on top (fp32 partials out and in)
constexpr int kShareMin = 16, kShareCost = 24;

struct alignas(64) HeadMaps { CUtensorMap a, a_rows, b; };

// How the tiles are dealt out.  Whole rounds of pairs take a tile each, in groups of row tiles (rows fastest) whose
// operands stay in L2 while the columns pass; the tiles of the last, partial round are shared out over their reduction,
// so that no pair is idle in it: the number of shares with the least rounds x (k-blocks + what a share costs).
struct Plan {
  int m_tiles, n_tiles, group, k_blocks;
  int whole, shares, items;          // tiles taken whole, shares of each other tile, items altogether
};
__device__ __forceinline__ Plan make_plan(int rows, int n_tiles, int k_blocks, int pairs, int most_items, bool split) {
  Plan t;
  t.m_tiles = (rows + kTile - 1) / kTile;
  t.n_tiles = n_tiles;
  t.k_blocks = k_blocks;
  const long long slice = (long long)kTile * k_blocks * kBK * 2;
  const int fit = (int)((40ll << 20) / slice);
  if (fit >= t.m_tiles) t.group = max(t.m_tiles, 1);
  else if (fit >= 8) { const int groups = (t.m_tiles + fit - 1) / fit; t.group = (t.m_tiles + groups - 1) / groups; }
  else t.group = 8;
  const int tiles = t.m_tiles * n_tiles, rest = tiles % pairs;
  t.whole = tiles;
  t.shares = 1;
  if (split && rest) {
    int best = k_blocks;
    for (int s = 2; s <= kHeadMaxShares && s * kShareMin <= k_blocks && s * rest <= most_items; ++s) {
      const int cost = (rest * s + pairs - 1) / pairs * ((k_blocks + s - 1) / s + kShareCost);
      if (cost < best) { best = cost; t.shares = s; }
    }
    if (t.shares > 1) t.whole = tiles - rest;
  }
  t.items = t.whole + (tiles - t.whole) * t.shares;
  return t;
}
struct Item { int m0, n0, kb0, kb1, tile, share; };   // tile: index among the shared tiles, -1 for a whole one
__device__ __forceinline__ Item item_at(const Plan& t, int i) {
  Item it;
  it.kb0 = 0; it.kb1 = t.k_blocks;
  it.tile = -1; it.share = 0;
  int tile = i;
  if (i >= t.whole && t.shares > 1) {
    it.tile = (i - t.whole) / t.shares;
    it.share = (i - t.whole) - it.tile * t.shares;
    it.kb0 = (int)((long long)it.share * t.k_blocks / t.shares);
    it.kb1 = (int)((long long)(it.share + 1) * t.k_blocks / t.shares);
    tile = t.whole + it.tile;
  }
  const int per_group = t.group * t.n_tiles;
  const int g = tile / per_group, in = tile - g * per_group;
  const int rows = min(t.group, t.m_tiles - g * t.group);
  const int col = in / rows;
  it.m0 = (g * t.group + in - col * rows) * kTile;
  it.n0 = col * kTile;
  return it;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// One row of 128 logits, in registers, by one thread: the listed ones are put aside, the others become exponentials.
template <bool GRAD, bool CAP>
__device__ __forceinline__ void logits_row(const HeadArgs& p, float (&x)[kHeadCols], int n0, int row, bool live) {
  constexpr int kChunks = kHeadCols / 32;
  const int token = live ? p.row_token[p.piece0 + row] : 0;
  const int32_t* list = p.list + (size_t)token * p.top;
  // the first listed column that may be among these
  int at = 0;
  if (live) {
    int hi = p.top;
    while (at < hi) {
      const int mid = (at + hi) >> 1;
      if (list[mid] < n0) at = mid + 1;
      else hi = mid;
    }
  }
  float* z = p.z_listed + (size_t)row * p.top + at;
  const float factor = p.logit_factor, cap_out = p.cap_out, to2 = p.to2;
  int next = live && at < p.top ? list[at] : kHeadNone;
  uint32_t dead[kChunks];       // a bit for each column that is listed or behind the vocabulary
  float most = -INFINITY;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int col = n0 + 32 * c;
    uint32_t named = 0;
    while (next < col + 32) {
      named |= 1u << (next - col);
      ++at;
      next = at < p.top ? list[at] : kHeadNone;
    }
    __syncwarp();
    if (named) {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (named >> j & 1) {
          const float raw = x[32 * c + j] * factor;
          *z++ = CAP ? tanhf(raw) * cap_out : raw;
        }
    }
    __syncwarp();
    dead[c] = named | (p.vocab - col >= 32 ? 0u : ~((1u << max(p.vocab - col, 0)) - 1u));
    if (__any_sync(0xffffffffu, dead[c])) {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (!(dead[c] >> j & 1)) most = fmaxf(most, x[32 * c + j]);
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j) most = fmaxf(most, x[32 * c + j]);
    }
  }
  most *= factor;
  if (CAP) most = tanhf(most) * cap_out;
  const float r = most == -INFINITY ? 0.f : kHeadStep * rintf(most * (1.4426950408889634f / kHeadStep));
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  bf16* e = reinterpret_cast<bf16*>(p.e) + (size_t)row * p.pitch + n0;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const bool any = __any_sync(0xffffffffu, dead[c]);
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      float& v = x[32 * c + j];
      float ex, slope = 1.f;
      if (CAP) {
        const float t = tanhf(v * factor);
        ex = exp2_fast(fmaf(t, to2, -r));
        slope = (1.f - t) * (1.f + t);
      } else {
        ex = exp2_fast(fmaf(v, to2, -r));
      }
      if (any && (dead[c] >> j & 1)) ex = 0.f;
      sum[j & 3] += ex;
      v = CAP ? ex * slope : ex;
    }
    if (GRAD && live) {
#pragma unroll
      for (int j = 32 * c; j < 32 * c + 32; j += 8)
        if (n0 + j < p.pitch)
          *reinterpret_cast<uint4*>(e + j) = make_uint4(pack_bf16(x[j], x[j + 1]), pack_bf16(x[j + 2], x[j + 3]),
                                                        pack_bf16(x[j + 4], x[j + 5]), pack_bf16(x[j + 6], x[j + 7]));
    }
  }
  if (live && n0 < p.vocab)
    p.stats[(size_t)row * p.col_tiles + n0 / kHeadCols] = make_float2(r, (sum[0] + sum[1]) + (sum[2] + sum[3]));
}

// 32 columns of one row of d_x
__device__ __forceinline__ void grad_chunk(const HeadArgs& p, bf16* out, float by, bool none, int col, uint32_t (&v)[32]) {
  if (none) {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = 0u;
  }
#pragma unroll
  for (int j = 0; j < 32; j += 8)
    if (col + j < p.d)
      *reinterpret_cast<uint4*>(out + col + j) =
          make_uint4(pack_bf16(by * __uint_as_float(v[j]), by * __uint_as_float(v[j + 1])),
                     pack_bf16(by * __uint_as_float(v[j + 2]), by * __uint_as_float(v[j + 3])),
                     pack_bf16(by * __uint_as_float(v[j + 4]), by * __uint_as_float(v[j + 5])),
                     pack_bf16(by * __uint_as_float(v[j + 6]), by * __uint_as_float(v[j + 7])));
}

enum { kLogits = 0, kLogitsGrad = 1, kLogitsCap = 2, kLogitsCapGrad = 3, kGrad = 4 };

template <int MODE>
__global__ void __launch_bounds__(threads_of(MODE == kGrad), 1) head_tc_kernel(const __grid_constant__ HeadArgs p,
                                                              const __grid_constant__ HeadMaps maps) {
  constexpr bool kToX = MODE == kGrad;                    // the second product: B is [K, N]
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * kStageBytes);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const uint32_t smem_base = smem_u32(smem), bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (kStages + s); };
  auto tfull_bar = [&](int b) { return bar_base + 8u * (2 * kStages + b); };
  auto tempty_bar = [&](int b) { return bar_base + 8u * (2 * kStages + 2 + b); };

  let_next_start();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 2 * result_warps(kToX)); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tmap(&maps.a); prefetch_tmap(&maps.a_rows); prefetch_tmap(&maps.b);
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                    // the peer's barriers exist before anything signals them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  wait_for_last();

  const int rows = head_rows_here(p);
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const Plan plan = kToX ? make_plan(rows, (p.d + kTile - 1) / kTile, (p.vocab + kBK - 1) / kBK, pairs, p.part_items, true)
                         : make_plan(rows, (p.vocab + kTile - 1) / kTile, (p.d + kBK - 1) / kBK, pairs, 0, false);

  if (warp == 0) {
    // ---------------- loads (both CTAs, each its own halves) ----------------
    if (lane == 0) {
      // where every token counts, x itself holds the rows
      const bool direct = kToX || p.state->counted == p.tokens;
      const CUtensorMap* am = direct ? &maps.a : &maps.a_rows;
      const int row0 = kToX || !direct ? 0 : p.piece0;
      uint32_t it = 0;
      bool ok = true;
      for (int i = pair; i < plan.items && ok; i += pairs) {
        const Item t = item_at(plan, i);
        const int m0 = row0 + t.m0 + (int)rank * 128, n0 = t.n0 + (int)rank * 128;
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const int st = it % kStages;
          if (!mbar_wait(empty_bar(st), ((it / kStages) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t a_dst = smem_base + st * kStageBytes, b_dst = a_dst + kABytes;
          const uint32_t bar = map_to_cta(full_bar(st), 0);
          if (leader) mbar_expect_tx(full_bar(st), 2 * kStageBytes);
          tma_load_2d_pair(a_dst, am, bar, kb * kBK, m0);
          if (kToX) {
            tma_load_2d_pair(b_dst, &maps.b, bar, n0, kb * kBK);
            tma_load_2d_pair(b_dst + kBK * 128, &maps.b, bar, n0 + 64, kb * kBK);
          } else {
            tma_load_2d_pair(b_dst, &maps.b, bar, kb * kBK, n0);
          }
        }
      }
      if (!ok) {
        *abort_flag = 1;
        atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
      }
    }
  } else if (warp == 1) {
    // ---------------- products (leader) ----------------
    if (lane == 0 && leader) {
      const uint32_t idesc = make_idesc_m(256, kTile, 0, kToX ? 1 : 0);
      uint32_t it = 0, count = 0;
      bool ok = true;
      for (int i = pair; i < plan.items && ok; i += pairs) {
        const Item t = item_at(plan, i);
        for (int k0 = t.kb0; k0 < t.kb1 && ok; k0 += kToX ? plan.k_blocks : kSpan, ++count) {
          const int k1 = kToX ? t.kb1 : min(k0 + kSpan, t.kb1);
          const uint32_t buf = count & 1u, use = count >> 1;
          if (!mbar_wait(tempty_bar(buf), (use & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t acc = tmem_base + buf * kTile;
          for (int kb = k0; kb < k1; ++kb, ++it) {
            const int st = it % kStages;
            if (!mbar_wait(full_bar(st), (it / kStages) & 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t a_addr = smem_base + st * kStageBytes, b_addr = a_addr + kABytes;
#pragma unroll
            for (int k = 0; k < kBK / kUmmaK; ++k) {
              const uint64_t ad = make_desc(a_addr + k * (kUmmaK * 2), 16, 1024);
              const uint64_t bd = kToX ? make_desc(b_addr + k * (kUmmaK * 128), kBK * 128, 1024)
                                       : make_desc(b_addr + k * (kUmmaK * 2), 16, 1024);
              umma_bf16_pair(acc, ad, bd, idesc, kb > k0 || k > 0);
            }
            umma_commit_pair(empty_bar(st), 3);
          }
          if (ok) umma_commit_pair(tfull_bar(buf), 3);
        }
      }
      if (!ok) {
        *abort_flag = 1;
        atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
      }
    }
  } else {
    // ---------------- results (both CTAs, a row per thread) ----------------
    const int q = warp & 3;
    uint32_t count = 0;
    bool ok = true;
    for (int i = pair; i < plan.items && ok; i += pairs) {
      const Item t = item_at(plan, i);
      const int row = t.m0 + (int)rank * 128 + q * 32 + lane;
      const bool live = row < rows;
      if constexpr (!kToX) {
        // The tensor core cuts off what a sum has behind its 24 bits, at every step of 16 products: over a whole row that
        // is a few 2^-20 of the logit, always towards zero.  So a sum starts anew every kSpan k-blocks, and the parts are
        // added here, rounded to nearest.
        const int half = (warp - 2) >> 2;
        float x[kHeadCols];
#pragma unroll
        for (int j = 0; j < kHeadCols; ++j) x[j] = 0.f;
        for (int k0 = 0; k0 < plan.k_blocks; k0 += kSpan, ++count) {
          const uint32_t buf = count & 1u, use = count >> 1;
          if (!__all_sync(0xffffffffu, mbar_wait(tfull_bar(buf), use & 1u, abort_flag))) { ok = false; break; }
          tc_fence_after();
          const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + buf * kTile + half * kHeadCols;
#pragma unroll
          for (int c = 0; c < kHeadCols; c += 32) {
            uint32_t v[32];
            tmem_ld32(acc + c, v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) x[c + j] += __uint_as_float(v[j]);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(map_to_cta(tempty_bar(buf), 0));
        }
        if (!ok) break;
        logits_row<(MODE & 1) != 0, (MODE & 2) != 0>(p, x, t.n0 + half * kHeadCols, row, live);
      } else {
        const uint32_t buf = count & 1u, use = count >> 1;
        ++count;
        if (!__all_sync(0xffffffffu, mbar_wait(tfull_bar(buf), use & 1u, abort_flag))) { ok = false; break; }
        tc_fence_after();
        const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + buf * kTile;
        float by = 0.f;
        bool none = false;                               // a token that is left out, where the rows have such
        bf16* out = nullptr;
        if (live) {
          const int token = p.row_token[p.piece0 + row];
          by = p.row_scale[row];
          none = p.token_row[token] < 0;
          out = reinterpret_cast<bf16*>(p.d_x) + (size_t)token * p.dx_stride;
        }
        if (t.tile >= 0) {
          // a share's partial sums, [chunk of 32 columns][4 columns][lane]: a warp's accesses cover 512 bytes at a time.
          // The warp that completes the tile adds them up in the shares' order, whoever it is.
          const size_t slab = (size_t)128 * kTile;
          const size_t mine = (size_t)q * 32 * kTile + (size_t)lane * 4;
          const float* first = p.part + ((size_t)t.tile * plan.shares * 2 + rank) * slab + mine;
          float* to = p.part + ((size_t)(t.tile * plan.shares + t.share) * 2 + rank) * slab + mine;
          for (int c = 0; c < kTile; c += 32) {
            uint32_t v[32];
            tmem_ld32(acc + c, v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; ++j)
              *reinterpret_cast<uint4*>(to + (c / 32 * 8 + j) * 128) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          }
          tc_fence_before();
          __threadfence();
          __syncwarp();
          int* counter = p.counters + (t.tile * 2 + (int)rank) * 4 + q;
          int seen = 0;
          if (lane == 0) {
            mbar_arrive_cluster(map_to_cta(tempty_bar(buf), 0));
            seen = atomicAdd(counter, 1);
          }
          seen = __shfl_sync(0xffffffffu, seen, 0);
          if (seen == plan.shares - 1) {
            __threadfence();
            for (int c = 0; c < kTile; c += 32) {
              float4 sum[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) sum[j] = make_float4(0.f, 0.f, 0.f, 0.f);
              for (int s = 0; s < plan.shares; s += 2) {
                float4 w[2][8];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                  for (int j = 0; j < 8; ++j)
                    w[h][j] = s + h < plan.shares
                                  ? __ldcg(reinterpret_cast<const float4*>(first + (size_t)(s + h) * 2 * slab + (c / 32 * 8 + j) * 128))
                                  : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                  for (int j = 0; j < 8; ++j) {
                    sum[j].x += w[h][j].x; sum[j].y += w[h][j].y; sum[j].z += w[h][j].z; sum[j].w += w[h][j].w;
                  }
              }
              uint32_t v[32];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                v[4 * j] = __float_as_uint(sum[j].x); v[4 * j + 1] = __float_as_uint(sum[j].y);
                v[4 * j + 2] = __float_as_uint(sum[j].z); v[4 * j + 3] = __float_as_uint(sum[j].w);
              }
              if (live) grad_chunk(p, out, by, none, t.n0 + c, v);
            }
            if (lane == 0) *counter = 0;                 // ready for the next piece
          }
          continue;
        }
        for (int c = 0; c < kTile; c += 32) {
          uint32_t v[32];
          tmem_ld32(acc + c, v);
          tmem_ld_wait();
          if (live) grad_chunk(p, out, by, none, t.n0 + c, v);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_to_cta(tempty_bar(buf), 0));
      }
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      atomicExch(&p.state->status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
    }
  }

  __syncthreads();
  if (*abort_flag) {
    for (int i = 0; i < 200; ++i) __nanosleep(5000);     // let copies that may still be in flight land
  }
  tc_fence_before();
  cluster_sync_all();                                    // neither CTA leaves while its peer may still touch it
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

template <int MODE>
cudaError_t launch(const HeadArgs& p, const HeadMaps& maps, long long most_items, cudaStream_t st) {
  static bool done[64] = {false};
  cudaError_t e = allow_smem(head_tc_kernel<MODE>, kSmemBytes, done);
  if (e != cudaSuccess) return e;
  const int pairs = (int)(most_items < head_pairs() ? (most_items > 0 ? most_items : 1) : head_pairs());
  return launch_behind_in_clusters(2, head_tc_kernel<MODE>, (unsigned)(2 * pairs), threads_of(MODE == kGrad), kSmemBytes, st, p, maps);
}

}  // namespace

int head_pairs() {
  static int sms[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 74;
  if (sms[dev] == 0) {
    int n = 0;
    sms[dev] = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 1 ? n : 148;
  }
  return sms[dev] / 2;
}

cudaError_t launch_head_logits_tc(const HeadArgs& p, cudaStream_t st) {
  HeadMaps m;
  if (!tc_encode_2d(&m.a, p.x, p.tokens, p.d, p.x_stride, 128, kBK) ||
      !tc_encode_2d(&m.a_rows, p.x_rows, p.piece, p.d, p.d, 128, kBK) ||
      !tc_encode_2d(&m.b, p.w, p.vocab, p.d, p.w_stride, 128, kBK))
    return cudaErrorInvalidValue;
  const long long items = (long long)((p.piece + kTile - 1) / kTile) * ((p.vocab + kTile - 1) / kTile);
  if (p.softcap > 0.f) return p.d_x ? launch<kLogitsCapGrad>(p, m, items, st) : launch<kLogitsCap>(p, m, items, st);
  return p.d_x ? launch<kLogitsGrad>(p, m, items, st) : launch<kLogits>(p, m, items, st);
}

cudaError_t launch_head_grad_tc(const HeadArgs& p, cudaStream_t st) {
  HeadMaps m;
  if (!tc_encode_2d(&m.a, p.e, p.piece, p.vocab, p.pitch, 128, kBK) ||
      !tc_encode_2d(&m.b, p.w, p.vocab, p.d, p.w_stride, kBK, 64))
    return cudaErrorInvalidValue;
  m.a_rows = m.a;
  return launch<kGrad>(p, m, head_pairs(), st);
}

}  // namespace mixlora
