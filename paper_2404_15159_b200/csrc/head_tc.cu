// The two products of the head's losses on the tensor cores (tcgen05, TMEM, TMA; bf16 operands, fp32 accumulation).
//
//   logits   x [rows, d] . w [vocab, d]^T   per half a tile's columns: R, S, the listed logits and, for a gradient, E
//   grad     E [rows, vocab] . w [vocab, d]  times the row's A scale / temperature weight / normalizer, to the row's token
//
// Pairs of CTAs work on 256 x 256 tiles (cta_group::2, 128 rows of the accumulator and half of B's columns each; the logits'
// tiles may be narrower, see head_cols), one persistent pair on two SMs; warp 0 loads, warp 1 of the leader issues the
// products, warps 2 to 9 take finished sums into registers, 128 columns of one row a thread, and turn them into results
// while the next sums are under way.  The number of rows is read on the device: tokens without a label take no part.
//
// The tensor core cuts off what a sum has behind its 24 bits, at every step of 16 products: over 4096 of them that is a few
// 2^-20 of a logit, always towards zero.  So a sum starts anew every few spans of k-blocks, and the parts are added up in
// registers, rounded to nearest; and every span of the logits has a partner that goes the other way (see Spans).
//
// Measured on a B200, 8192 rows, 32000 columns, width 4096: logits 1.51 ms, gradient 1.45 ms in short runs (1.42 and
// 1.48 PFLOP/s, tensor pipe 79 and 90 % active at 1.6 and 1.5 GHz under the power cap), 3.41 ms a call one after another
// (1.26 PFLOP/s; the library's own dense product in such a loop: 1.38).  512 rows: 116 and 98 us (four rounds of tiles for
// 3.4; tiles that are narrower wait for their operands as long).
//
// In the fp32 mode (PARTS = 3) an operand is the sum of three bf16 values that hold its 24 bits, and the six products of
// parts that matter at 2^-24 are added up, the small ones first: exact to fp32's own rounding, at a sixth of the rate, which
// is still three times that of the fp32 pipes.
#include <cuda.h>
#include <math.h>

#include "head.cuh"
#include "tc_ptx.cuh"

namespace mixlora {
namespace {

using namespace tc;
constexpr int kBK = 64, kUmmaK = 16, kTile = kHeadTile;
constexpr int kResultWarps = 8, kThreads = 64 + 32 * kResultWarps;
constexpr uint32_t kHalf = 128 * kBK * 2;                 // bytes of one CTA's part of an operand, one k-block
constexpr uint32_t kTmemCols = 512;
template <bool TO_X, int PARTS> struct Form {
  static constexpr int kStages = PARTS == 1 ? 6 : 2;
  static constexpr uint32_t kStage = PARTS * 2 * kHalf;
  static constexpr uint32_t kSmem = kStages * kStage + 1024 + 256;
  // k-blocks of a span.  Its end costs the tensor core about 360 cycles, since the sums are read from the memory that it works
  // in: with spans of 4 / 8 / 16 k-blocks throughout 4096 tokens of width 4096 take 963 / 867 / 829 us.  The gradient's product is
  // rounded to bf16 in the end, where 512 steps are nothing, and with parts a k-block is 24 steps already.
  static constexpr int kSpan = PARTS == 3 ? 1 : (TO_X ? 128 : 16);
  static constexpr bool kTurns = !TO_X && PARTS == 1;
  // a share of a split reduction keeps at least this many k-blocks, and costs this many on top (partial sums out and in): with
  // a cost of 8 or 12, which takes nine shares where 24 takes four, 333 tokens of width 2048 took 135 us instead of 129
  static constexpr int kShareMin = PARTS == 1 ? 16 : 3, kShareCost = PARTS == 1 ? 24 : 4;
};
// The spans of a tile's sums, one after another: the one that starts at k-block k0 ends at k1.
//
// Where spans turn around, up to four make a group: the first two, one in either accumulator, add their products up from
// zero, and the other two go on in the same accumulators with their products subtracted, back to about zero where a row's
// products lean one way.  On the way up the cut takes from the first sum a, on the way down from a - b, which adds it to
// b: a + b = 2 a - (a - b) has lost on one way what it won on the other.  On logits whose products lean by 0.3 of their spread, as a
// sure token's with its label, width 4096: too small by 8.9 units of 2^-23 with spans of 16 k-blocks that do not turn, by 2.0 with
// spans of 4 (which take 15 % longer), by 0.3 with spans of 16 that do (which take 1 to 3 %: adding to what is there at a
// span's start, and the change of sign), with a spread of 0.95 (fp32's own products: 0 and 0.5).  A span without a partner has 4
// k-blocks at most.  Of products of one sign the cut at each product's own last bits remains: 9.8 units.
constexpr int kLeastSpan = 4;
template <bool TO_X, int PARTS> struct Spans {
  using F = Form<TO_X, PARTS>;
  int k1 = 0, end = 0, each = 0, turn = 0;
  bool back = false;                  // the products are subtracted
  float factor = 1.f;                 // of what the accumulator holds at the span's end
  __device__ __forceinline__ void start(int k0, int kb1) {
    if constexpr (!F::kTurns) {
      k1 = min(k0 + F::kSpan, kb1);
    } else {
      if (k0 >= end) {
        end = min(k0 + 4 * F::kSpan, kb1);
        each = max((end - k0 + 3) / 4, kLeastSpan);
        turn = k0 + 2 * each;
      }
      back = k0 >= turn;
      factor = back ? -1.f : (k0 + 2 * each < end ? 2.f : 1.f);
      k1 = min(k0 + each, end);
    }
  }
};
// the six products of parts, small ones first
__device__ constexpr int kPartOfA[6] = {2, 0, 1, 1, 0, 0}, kPartOfB[6] = {0, 2, 1, 0, 1, 0};
constexpr int kCorners = 16, kCornerSums = 32 * kHeadCols, kTileSums = kCorners * kCornerSums, kAddThreads = 256;
struct alignas(64) HeadMaps { CUtensorMap a, a_rows, b; };

// 32 bytes, at such a boundary, with one instruction: a warp's rows are far apart, and every instruction visits all of them
__device__ __forceinline__ void store_32(void* to, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// How the tiles are dealt out.  Whole rounds of pairs take a tile each, in groups of row tiles (rows fastest) whose
// operands stay in L2 while the columns pass; the tiles of the last, partial round are shared out over their reduction,
// so that no pair is idle in it: the number of shares with the least rounds x (k-blocks + what a share costs).
struct Plan {
  int m_tiles, n_tiles, group, k_blocks;
  int whole, shares, items;          // tiles taken whole, shares of each other tile, items altogether
};
template <bool TO_X, int PARTS>
__device__ __forceinline__ Plan make_plan(int rows, int n_tiles, int k_blocks, int pairs, int most_items) {
  Plan t;
  t.m_tiles = (rows + kTile - 1) / kTile;
  t.n_tiles = n_tiles;
  t.k_blocks = k_blocks;
  const long long slice = (long long)kTile * k_blocks * kBK * 2 * PARTS;
  const int fit = (int)((40ll << 20) / slice);
  if (fit >= t.m_tiles) t.group = max(t.m_tiles, 1);
  else if (fit >= 8) { const int groups = (t.m_tiles + fit - 1) / fit; t.group = (t.m_tiles + groups - 1) / groups; }
  else t.group = 8;
  const int tiles = t.m_tiles * n_tiles, rest = tiles % pairs;
  t.whole = tiles;
  t.shares = 1;
  if (TO_X && rest) {
    // in whole numbers, costs times shares compared crosswise: the kernel that adds the shares up has to come to the same plan
    int best = k_blocks, rounds = 1, items = rest;
#pragma unroll
    for (int s = 2; s <= kHeadMaxShares; ++s) {
      items += rest;
      rounds += items > rounds * pairs;                    // of `pairs` items, rounded up: rest < pairs
      if (s * Form<TO_X, PARTS>::kShareMin > k_blocks || items > most_items) continue;
      const int cost = rounds * (k_blocks + s * Form<TO_X, PARTS>::kShareCost);
      if (cost * t.shares < best * s) { best = cost; t.shares = s; }
    }
    if (t.shares > 1) t.whole = tiles - rest;
  }
  t.items = t.whole + (tiles - t.whole) * t.shares;
  return t;
}
struct Item { int m0, n0, kb0, kb1, tile, share; };   // tile: index among the shared tiles, -1 for a whole one
__device__ __forceinline__ Item item_at(const Plan& t, int i, int width) {
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
  it.n0 = col * width;
  return it;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// One row of up to 128 logits, in registers, by one thread: the listed ones are put aside, the others become exponentials.
// A cap, or an exponential, would make a number of a product that is infinite: 0 times it is added to what the row leaves.
template <bool GRAD, bool CAP, int PARTS>
__device__ __forceinline__ void logits_row(const HeadArgs& p, float (&x)[kHeadCols], int n0, int row, bool live) {
  constexpr int kChunk = 16, kChunks = kHeadCols / kChunk;
  const int cols = p.cols;
  const int token = live ? head_token(p, row) : 0;
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
  float most = -INFINITY, far = 0.f;       // far: the largest magnitude
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    if (c * kChunk >= cols) break;
    const int col = n0 + kChunk * c;
    uint32_t named = 0;
    while (next < col + kChunk) {
      named |= 1u << (next - col);
      ++at;
      next = at < p.top ? list[at] : kHeadNone;
    }
    __syncwarp();
    if (named) {
#pragma unroll
      for (int j = 0; j < kChunk; ++j)
        if (named >> j & 1) {
          const float raw = x[kChunk * c + j] * factor;
          *z++ = fmaf(raw, 0.f, CAP ? tanhf(raw) * cap_out : raw);
        }
    }
    __syncwarp();
    dead[c] = named | (p.vocab - col >= kChunk ? 0u : ~((1u << max(p.vocab - col, 0)) - 1u));
    if (__any_sync(0xffffffffu, dead[c])) {
#pragma unroll
      for (int j = 0; j < kChunk; ++j)
        if (!(dead[c] >> j & 1)) {
          most = fmaxf(most, x[kChunk * c + j]);
          far = fmaxf(far, fabsf(x[kChunk * c + j]));
        }
    } else {
#pragma unroll
      for (int j = 0; j < kChunk; ++j) {
        most = fmaxf(most, x[kChunk * c + j]);
        far = fmaxf(far, fabsf(x[kChunk * c + j]));
      }
    }
  }
  most *= factor;
  if (CAP) most = tanhf(most) * cap_out;
  const float r = most == -INFINITY ? 0.f : kHeadStep * rintf(most * (1.4426950408889634f / kHeadStep));
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  bf16* e = reinterpret_cast<bf16*>(p.e) + (size_t)row * p.pitch + n0;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    if (c * kChunk >= cols) break;
    const bool any = __any_sync(0xffffffffu, dead[c]);
#pragma unroll
    for (int j = 0; j < kChunk; ++j) {
      float& v = x[kChunk * c + j];
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
    if (GRAD && live && n0 + kChunk * c < p.pitch) {
#pragma unroll
      for (int n = 0; n < PARTS; ++n) {
        uint32_t out[kChunk / 2];
#pragma unroll
        for (int j = 0; j < kChunk; j += 2) {
          float &lo = x[kChunk * c + j], &up = x[kChunk * c + j + 1];
          if (PARTS == 3 && n == 0) {                      // a part, and what it leaves for the next
            const float a = head_cut(lo), b = head_cut(up);
            out[j / 2] = pack_bf16(a, b);
            lo -= a;
            up -= b;
          } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(lo, up);
            out[j / 2] = *reinterpret_cast<const uint32_t*>(&h);
            if (PARTS == 3 && n == 1) {
              const float2 f = __bfloat1622float2(h);
              lo -= f.x;
              up -= f.y;
            }
          }
        }
        store_32(e + n * p.e_part + kChunk * c, out);
      }
    }
  }
  if (live && n0 < p.vocab)
    p.stats[(size_t)row * p.col_tiles + n0 / cols] = make_float2(r, fmaf(far, 0.f, (sum[0] + sum[1]) + (sum[2] + sum[3])));
}

// One row of 128 sums of the gradient's product.  Where a tile's reduction is shared, the sums go to `part`, corner by corner
// (32 rows x 128 columns) as [4 columns][row] so that a warp's accesses cover 512 bytes.
template <int PARTS>
__device__ __forceinline__ void grad_row(const HeadArgs& p, float (&x)[kHeadCols], const Plan& plan, const Item& t, int corner,
                                         int n0, int row, bool live) {
  if (t.tile >= 0) {
    float* to = p.part + (size_t)(t.tile * plan.shares + t.share) * kTileSums + corner * kCornerSums + (threadIdx.x & 31) * 4;
#pragma unroll
    for (int j = 0; j < kHeadCols; j += 4)
      *reinterpret_cast<float4*>(to + j * 32) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
    return;
  }
  if (!live) return;
  const int token = head_token(p, row);
  const float by = p.row_scale[row];
  const bool none = head_left_out(p, token);
#pragma unroll
  for (int j = 0; j < kHeadCols; ++j) x[j] = none ? 0.f : x[j] * by;
  if constexpr (PARTS == 1) {
    bf16* out = reinterpret_cast<bf16*>(p.d_x) + (size_t)token * p.dx_stride + n0;
#pragma unroll
    for (int j = 0; j < kHeadCols; j += 8)
      if (n0 + j < p.d)
        *reinterpret_cast<uint4*>(out + j) = make_uint4(pack_bf16(x[j], x[j + 1]), pack_bf16(x[j + 2], x[j + 3]),
                                                        pack_bf16(x[j + 4], x[j + 5]), pack_bf16(x[j + 6], x[j + 7]));
  } else {
    float* out = reinterpret_cast<float*>(p.d_x) + (size_t)token * p.dx_stride + n0;
#pragma unroll
    for (int j = 0; j < kHeadCols; j += 4)
      if (n0 + j < p.d) *reinterpret_cast<float4*>(out + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
  }
}

// The shared tiles' rows of d_x: a block adds up the shares of one corner, in their order, and turns it for the way out.  In
// a launch of its own all SMs take part; where the CTA that finished a tile last added it up, 12 shares of 2 MB took it 20 us.
template <int PARTS>
__global__ void __launch_bounds__(kAddThreads) head_add_kernel(HeadArgs p, int pairs) {
  let_next_start();
  wait_for_last();
  __shared__ float turn[32][kHeadCols + 4];
  const int rows = head_rows_here(p);
  const Plan plan = make_plan<true, PARTS>(rows, (p.d + kTile - 1) / kTile, (p.vocab + kBK - 1) / kBK, pairs, p.part_items);
  const int tile = blockIdx.x / kCorners, corner = blockIdx.x - tile * kCorners;
  if (plan.shares == 1 || plan.whole + tile * plan.shares >= plan.items) return;
  const Item t = item_at(plan, plan.whole + tile * plan.shares, kTile);
  const int m0 = t.m0 + (corner >> 1) * 32, n0 = t.n0 + (corner & 1) * kHeadCols;
  if (m0 >= rows || n0 >= p.d) return;
  const float* from = p.part + (size_t)tile * plan.shares * kTileSums + corner * kCornerSums + threadIdx.x * 4;
  constexpr int kEach = kCornerSums / 4 / kAddThreads;
  float4 sum[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) sum[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int s = 0; s < plan.shares; ++s) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(from + s * kTileSums + i * kAddThreads * 4));
      sum[i].x += v.x; sum[i].y += v.y; sum[i].z += v.z; sum[i].w += v.w;
    }
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = threadIdx.x + i * kAddThreads;          // [4 columns][row]
    *reinterpret_cast<float4*>(&turn[at & 31][(at >> 5) * 4]) = sum[i];
  }
  __syncthreads();
  constexpr int kWide = PARTS == 1 ? 8 : 4;                // values of 16 bytes
  for (int i = threadIdx.x; i < kCornerSums / kWide; i += kAddThreads) {
    const int r = i / (kHeadCols / kWide), c = (i - r * (kHeadCols / kWide)) * kWide;
    if (m0 + r >= rows || n0 + c >= p.d) continue;
    const float by = p.row_scale[m0 + r];
    const int token = head_token(p, m0 + r);
    const size_t at = (size_t)token * p.dx_stride + n0 + c;
    if (head_left_out(p, token)) {
      uint4* to = PARTS == 1 ? reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(p.d_x) + at)
                             : reinterpret_cast<uint4*>(reinterpret_cast<float*>(p.d_x) + at);
      *to = make_uint4(0, 0, 0, 0);
      continue;
    }
    const float4 lo = *reinterpret_cast<const float4*>(&turn[r][c]);
    if constexpr (PARTS == 1) {
      const float4 up = *reinterpret_cast<const float4*>(&turn[r][c + 4]);
      *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(p.d_x) + at) =
          make_uint4(pack_bf16(by * lo.x, by * lo.y), pack_bf16(by * lo.z, by * lo.w), pack_bf16(by * up.x, by * up.y),
                     pack_bf16(by * up.z, by * up.w));
    } else {
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(p.d_x) + at) = make_float4(by * lo.x, by * lo.y, by * lo.z, by * lo.w);
    }
  }
}

template <bool TO_X, bool GRAD, bool CAP, int PARTS>
__global__ void __launch_bounds__(kThreads, 1) head_tc_kernel(const __grid_constant__ HeadArgs p,
                                                              const __grid_constant__ HeadMaps maps) {
  using F = Form<TO_X, PARTS>;
  constexpr int kStages = F::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kStages * F::kStage);
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
    for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 2 * kResultWarps); }
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

  if (!TO_X && p.few && blockIdx.x == 0 && threadIdx.x == 0) {
    p.state->status = 0;
    p.state->joined = 0;
  }
  const int rows = head_rows_here(p);
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int cols = TO_X ? kHeadCols : p.cols;              // half of a tile's columns
  const Plan plan = make_plan<TO_X, PARTS>(rows, ((TO_X ? p.d : p.vocab) + 2 * cols - 1) / (2 * cols),
                                           ((TO_X ? p.vocab : p.d) + kBK - 1) / kBK, pairs, p.part_items);

  if (warp == 0) {
    // ---------------- loads (both CTAs, each its own halves) ----------------
    if (lane == 0) {
      // where every token counts, x itself holds the rows (not its parts)
      const bool direct = !TO_X && PARTS == 1 && (p.few || p.state->counted == p.tokens);
      const CUtensorMap* am = direct ? &maps.a : &maps.a_rows;
      const int row0 = direct ? p.piece0 : 0;
      const uint32_t bytes = 2 * PARTS * (kHalf + cols * kBK * 2);      // of both CTAs' operands
      uint32_t it = 0;
      bool ok = true;
      for (int i = pair; i < plan.items && ok; i += pairs) {
        const Item t = item_at(plan, i, 2 * cols);
        const int m0 = row0 + t.m0 + (int)rank * 128, n0 = t.n0 + (int)rank * cols;
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const int st = it % kStages;
          if (!mbar_wait(empty_bar(st), ((it / kStages) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t a_dst = smem_base + st * F::kStage, b_dst = a_dst + PARTS * kHalf;
          const uint32_t bar = map_to_cta(full_bar(st), 0);
          if (leader) mbar_expect_tx(full_bar(st), bytes);
#pragma unroll
          for (int n = 0; n < PARTS; ++n) {
            tma_load_2d_pair(a_dst + n * kHalf, am, bar, kb * kBK, m0 + n * p.piece);
            if (TO_X) {
              tma_load_2d_pair(b_dst + n * kHalf, &maps.b, bar, n0, kb * kBK + n * p.vocab);
              tma_load_2d_pair(b_dst + n * kHalf + kHalf / 2, &maps.b, bar, n0 + 64, kb * kBK + n * p.vocab);
            } else {
              tma_load_2d_pair(b_dst + n * kHalf, &maps.b, bar, kb * kBK, n0 + n * p.vocab);
            }
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
      const uint32_t idesc = make_idesc_m(256, 2 * cols, 0, TO_X ? 1 : 0);
      constexpr uint32_t kNegateA = 1u << 13;
      uint32_t it = 0, count = 0;
      bool ok = true;
      for (int i = pair; i < plan.items && ok; i += pairs) {
        const Item t = item_at(plan, i, 2 * cols);
        Spans<TO_X, PARTS> span;
        for (int k0 = t.kb0; k0 < t.kb1 && ok; k0 = span.k1, ++count) {
          span.start(k0, t.kb1);
          const uint32_t buf = count & 1u, use = count >> 1;
          if (!mbar_wait(tempty_bar(buf), (use & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t acc = tmem_base + buf * kTile;
          for (int kb = k0; kb < span.k1; ++kb, ++it) {
            const int st = it % kStages;
            if (!mbar_wait(full_bar(st), (it / kStages) & 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t a_addr = smem_base + st * F::kStage, b_addr = a_addr + PARTS * kHalf;
#pragma unroll
            for (int c = PARTS == 1 ? 5 : 0; c < 6; ++c) {
              const uint32_t a_part = a_addr + kPartOfA[c] * kHalf, b_part = b_addr + kPartOfB[c] * kHalf;
#pragma unroll
              for (int k = 0; k < kBK / kUmmaK; ++k) {
                const uint64_t ad = make_desc(a_part + k * (kUmmaK * 2), 16, 1024);
                const uint64_t bd = TO_X ? make_desc(b_part + k * (kUmmaK * 128), kBK * 128, 1024)
                                         : make_desc(b_part + k * (kUmmaK * 2), 16, 1024);
                umma_bf16_pair(acc, ad, bd, span.back ? idesc | kNegateA : idesc,
                               span.back || kb > k0 || k > 0 || c > (PARTS == 1 ? 5 : 0));
              }
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
    const int q = warp & 3, half = (warp - 2) >> 2;      // the TMEM lanes that a warp may read go by its number
    uint32_t count = 0;
    bool ok = true;
    for (int i = pair; i < plan.items && ok; i += pairs) {
      const Item t = item_at(plan, i, 2 * cols);
      const int row = t.m0 + (int)rank * 128 + q * 32 + lane;
      const bool live = row < rows;
      float x[kHeadCols];
#pragma unroll
      for (int j = 0; j < kHeadCols; ++j) x[j] = 0.f;
      Spans<TO_X, PARTS> span;
      for (int k0 = t.kb0; k0 < t.kb1; k0 = span.k1, ++count) {
        span.start(k0, t.kb1);
        const uint32_t buf = count & 1u, use = count >> 1;
        if (!__all_sync(0xffffffffu, mbar_wait(tfull_bar(buf), use & 1u, abort_flag))) { ok = false; break; }
        tc_fence_after();
        const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + buf * kTile + half * cols;
#pragma unroll
        for (int c = 0; c < kHeadCols; c += 32) {
          if (c >= cols) break;                            // the last columns of 32 may be another half's, or nothing's
          uint32_t v[32];
          tmem_ld32(acc + c, v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j) x[c + j] = fmaf(__uint_as_float(v[j]), span.factor, x[c + j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_to_cta(tempty_bar(buf), 0));
      }
      if (!ok) break;
      const int n0 = t.n0 + half * cols;
      if constexpr (TO_X) grad_row<PARTS>(p, x, plan, t, (int)rank * 8 + q * 2 + half, n0, row, live);
      else logits_row<GRAD, CAP, PARTS>(p, x, n0, row, live);
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

template <bool TO_X, bool GRAD, bool CAP, int PARTS>
cudaError_t launch(const HeadArgs& p, const HeadMaps& maps, long long most_items, cudaStream_t st) {
  static bool done[64] = {false};
  constexpr auto kernel = head_tc_kernel<TO_X, GRAD, CAP, PARTS>;
  constexpr uint32_t kSmem = Form<TO_X, PARTS>::kSmem;
  cudaError_t e = allow_smem(kernel, kSmem, done);
  if (e != cudaSuccess) return e;
  const int pairs = (int)(most_items < head_pairs() ? (most_items > 0 ? most_items : 1) : head_pairs());
  return launch_behind_in_clusters(2, kernel, (unsigned)(2 * pairs), kThreads, kSmem, st, p, maps);
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
  return sms[dev] / 2 < kHeadMostPairs ? sms[dev] / 2 : kHeadMostPairs;
}

cudaError_t launch_head_logits_tc(const HeadArgs& p, cudaStream_t st) {
  HeadMaps m;
  const bool parts = p.parts == 3;
  if (!tc_encode_2d(&m.a_rows, p.x_rows, (long long)p.parts * p.piece, p.d, p.d, 128, kBK)) return cudaErrorInvalidValue;
  if (parts ? !tc_encode_2d(&m.b, p.w_parts, 3LL * p.vocab, p.d, p.d, p.cols, kBK)
            : !tc_encode_2d(&m.b, p.w, p.vocab, p.d, p.w_stride, p.cols, kBK) ||
                  !tc_encode_2d(&m.a, p.x, p.tokens, p.d, p.x_stride, 128, kBK))
    return cudaErrorInvalidValue;
  if (parts) m.a = m.a_rows;
  const long long items = (long long)((p.piece + kTile - 1) / kTile) * ((p.vocab + 2 * p.cols - 1) / (2 * p.cols));
  const bool cap = p.softcap > 0.f, grad = p.d_x != nullptr;
  if (parts) {
    if (cap) return grad ? launch<false, true, true, 3>(p, m, items, st) : launch<false, false, true, 3>(p, m, items, st);
    return grad ? launch<false, true, false, 3>(p, m, items, st) : launch<false, false, false, 3>(p, m, items, st);
  }
  if (cap) return grad ? launch<false, true, true, 1>(p, m, items, st) : launch<false, false, true, 1>(p, m, items, st);
  return grad ? launch<false, true, false, 1>(p, m, items, st) : launch<false, false, false, 1>(p, m, items, st);
}

cudaError_t launch_head_grad_tc(const HeadArgs& p, cudaStream_t st) {
  HeadMaps m;
  const bool parts = p.parts == 3;
  if (!tc_encode_2d(&m.a_rows, p.e, (long long)p.parts * p.piece, p.vocab, p.pitch, 128, kBK) ||
      !tc_encode_2d(&m.b, parts ? p.w_parts : p.w, (long long)p.parts * p.vocab, p.d, parts ? p.d : p.w_stride, kBK, 64))
    return cudaErrorInvalidValue;
  m.a = m.a_rows;
  const int pairs = head_pairs();
  const cudaError_t e = parts ? launch<true, true, false, 3>(p, m, pairs, st) : launch<true, true, false, 1>(p, m, pairs, st);
  if (e != cudaSuccess) return e;
  const unsigned blocks = (unsigned)((pairs - 1) * kCorners);     // less than a round of tiles is shared
  return parts ? launch_behind(head_add_kernel<3>, blocks, kAddThreads, 0, st, p, pairs)
               : launch_behind(head_add_kernel<1>, blocks, kAddThreads, 0, st, p, pairs);
}

}  // namespace mixlora
