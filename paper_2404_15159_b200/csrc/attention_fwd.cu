// Masked attention, forward, bf16, on the tensor cores.
//
//   s_ij = scale q_i . k_j          capped: s <- c tanh(s / c)          lowered with distance: s <- s - a_h |p_i - p_j|
//   o_i  = sum_j e^(s_ij - m_i) v_j / l_i,   l_i = sum_j e^(s_ij - m_i),   m_i = a running maximum,   lse_i = m_i + ln l_i
//
// over the keys that row i sees.
#include <cuda.h>
#include <string.h>

#include "attention.cuh"
#include "tc_ptx.cuh"

namespace mixlora {
namespace {
using namespace tc;

constexpr int kTile = 128;                       // keys per step, and query rows per half of a block's rows
constexpr int kThreads = 384;                    // two softmax groups of 4 warps; a group with the load and MMA warps
// A block starts with 168 registers a thread (384 x 168 = 64512); the softmax groups, whose threads hold 64 scores and
// their exponentials, take 208 and the third group keeps 88: (2 x 208 + 88) x 128 = 64512.
constexpr int kLoadWarp = 8, kMmaWarp = 9;       // and 10: one for each query half
constexpr int kTmemCols = 512;
constexpr float kRaise = 0x1p16f, kRetake = 0x1p24f;         // sums of p that move the running maximum, see below
template <int DP> constexpr int kStages = DP == 128 ? 5 : 8;
template <int DP> constexpr uint32_t kTileBytes = kTile * DP * 2;
template <int DP> constexpr uint32_t kSmemBytes = (2 + kStages<DP>) * kTileBytes<DP> + 320;

struct FwdParams {
  AttnArgs a;
  CUtensorMap q_map, k_map, v_map;
};

// One block per SM walks over (256 query rows, head) pairs, longest first: two halves of 128 rows against the sequence's
// key tiles.  The load warp streams K and V tiles through a ring and runs ahead into the next pair's Q and K while this
// one's results are written.  Each half has an MMA warp, which issues O += P V and then the next S = Q K^T, and four
// softmax warps, a row to a thread: while one half's products run the other half's exponentials are computed.
// S [128 x 128] sits in TMEM; P is written over it as bf16, from where the product reads it, so it never touches shared
// memory, and its first half is used while the second is computed.
//
// P is rounded to bf16, the tensor cores' operand type: half a step, 2^-8 of a weight.  The log-sum-exp comes from the
// sums of the unrounded values in fp32; O is divided by the sum of the rounded ones.
//
// The running maximum m stands for "large enough": p = 2^(s - m) is taken over the m of the tiles before, without
// waiting for this tile's maximum.  A tile whose p sum up to more than 2^16 raises m for the next one, and only a row's
// first keys, or p of 64 keys that sum up to more than 2^24, are taken again over their own maximum.  Scores capped at up to
// 2^96 either way (no distance term) start from m = 0 instead, unless a row's first p sum up to less than 2^-24.  So O stays
// below 2^40 |v| (2^23 tiles of 2^16, one of 2^24) and a row's largest p above 2^-30, which leaves v from 2^-80 to 2^80.
// m is a whole number in base 2, so that raising it rescales O and l exactly.
//
// A 128 x 128 tile costs 1024 cycles of the special-function unit (16 exponentials a cycle) and, at 128 values a head,
// 1024 of the tensor pipe; a half's chain of waiting for S, reading it, exponentials, P, product and next S takes about
// 3300, so the pipes are active for about half of the time each.  Measured: one sequence of 8192 rows, 32 heads of 128,
// causal, 523 us (1.05 PFLOP/s) alone and 605 to 625 one after another, where the power cap takes the clock to 1.58 GHz; 24
// documents in 5003 rows, 32 / 8 heads of 64, capped, 59 us.
template <int DP, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) attn_fwd_tc_kernel(const __grid_constant__ FwdParams p) {
  constexpr int NS = kStages<DP>;
  constexpr uint32_t TB = kTileBytes<DP>;
  constexpr int NB = DP / 64;                    // 64-value blocks of a head in a tile
  extern __shared__ __align__(1024) uint8_t smem[];          // the swizzle counts from 1024-byte boundaries
  const uint32_t q_base = smem_u32(smem), ring = q_base + 2 * TB;
  uint8_t* ctl = smem + (2 + NS) * TB;
  const uint32_t bars = smem_u32(ctl);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (NS + s); };
  auto q_bar = [&](int h) { return bars + 8u * (2 * NS + h); };
  auto s_bar = [&](int h) { return bars + 8u * (2 * NS + 2 + h); };
  auto p_bar = [&](int h) { return bars + 8u * (2 * NS + 4 + h); };      // and 16 bytes on, for the second half of P
  auto o_bar = [&](int h) { return bars + 8u * (2 * NS + 8 + h); };
  auto v_bar = [&](int h) { return bars + 8u * (2 * NS + 10 + h); };     // the first half of P has been used
  auto q_empty_bar = [&](int h) { return bars + 8u * (2 * NS + 12 + h); };
  auto o_empty_bar = [&](int h) { return bars + 8u * (2 * NS + 14 + h); };
  uint32_t* slot = reinterpret_cast<uint32_t*>(ctl + 8 * (2 * NS + 16));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(slot + 1);
  volatile int* turns = reinterpret_cast<volatile int*>(slot + 2);       // [2] tiles of both halves that each has reached

  const AttnArgs& a = p.a;
  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (threadIdx.x == 32) {
    for (int s = 0; s < NS; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 2); }
    for (int h = 0; h < 2; ++h) {
      mbar_init(q_bar(h), 1); mbar_init(s_bar(h), 1); mbar_init(o_bar(h), 1); mbar_init(v_bar(h), 1);
      mbar_init(p_bar(h), 4); mbar_init(p_bar(h) + 16u, 4); mbar_init(q_empty_bar(h), 1); mbar_init(o_empty_bar(h), 4);
    }
    *abort_flag = 0;
    turns[0] = turns[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kLoadWarp && lane == 0) { prefetch_tmap(&p.q_map); prefetch_tmap(&p.k_map); prefetch_tmap(&p.v_map); }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(slot), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(*slot);
  wait_for_last();                               // the plan
  TileWalk w(a.q_tiles, a.n_q_tiles, a.q_heads);
  // of the tile at hand: its rows, its key tiles, and those of them that a half of the rows needs
  auto rows_of = [&] { return min(2 * kTile, w.sq.lq - w.row0); };
  auto tiles_of = [&] {
    const int p0 = w.sq.shift + w.row0;
    return key_tiles<kTile>(w.sq, a.causal, a.window, p0, p0 + rows_of() - 1);
  };
  // Scores that are lowered with distance grow towards a row's own position, so then the last keys come first: m starts
  // near its end, where in ascending order nearly every tile would raise it and rescale O (2901 rows, window 500, capped,
  // 20 heads of 80: 48 us, and 41 in this order).
  auto tile_at = [&](const KeyTiles<kTile>& tiles, int i) { return tiles.at(BIAS ? tiles.count() - 1 - i : i); };
  auto half_tiles = [&](int h) {
    const int hr = min(kTile, rows_of() - h * kTile);
    if (hr <= 0) return KeyTiles<kTile>{0, 0, 0};
    const int p0 = w.sq.shift + w.row0 + h * kTile;
    return key_tiles<kTile>(w.sq, a.causal, a.window, p0, p0 + hr - 1);
  };

  if (warp >= kLoadWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kLoadWarp) {
      if (lane == 0) {
        bool ok = true;
        int used = 0, q_used[2] = {0, 0};          // ring slots and Q halves that have been filled
        while (ok && w.next()) {
          const int kvh = w.head / a.group;
          const KeyTiles<kTile> tiles = tiles_of();
          const int n = tiles.count();
          for (int h = 0; h < 2; ++h) {
            if (half_tiles(h).count() == 0) continue;
            if (!mbar_wait(q_empty_bar(h), (q_used[h] & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            ++q_used[h];
            mbar_expect_tx(q_bar(h), TB);
            for (int j = 0; j < NB; ++j)
              tma_load_3d(q_base + h * TB + j * (kTile * 128), &p.q_map, q_bar(h), j * 64, w.head,
                          w.sq.q0 + w.row0 + h * kTile);
          }
          for (int i = 0; i < 2 * n && ok; ++i, ++used) {      // K and V of a tile in turn
            const int st = used % NS;
            if (!mbar_wait(empty_bar(st), ((used / NS) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            mbar_expect_tx(full_bar(st), TB);
            const CUtensorMap* map = (i & 1) ? &p.v_map : &p.k_map;
            for (int j = 0; j < NB; ++j)
              tma_load_3d(ring + st * TB + j * (kTile * 128), map, full_bar(st), j * 64, kvh,
                          w.sq.k0 + tile_at(tiles, i >> 1) * kTile);
          }
        }
        if (!ok) {
          *abort_flag = 1;
          if (a.status) atomicExch(a.status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
        }
      }
    } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
      const int h = warp - kMmaWarp;
      const uint32_t idesc_s = make_idesc(kTile, 0, 0), idesc_o = make_idesc(DP, 0, 1);
      const uint32_t t_s = tmem + h * kTile, t_o = tmem + 2 * kTile + h * DP;
      const bool one = elect_one();
      int base = 0;                                // ring slots of the tiles before
      int q_used = 0, done = 0;                    // tiles of Q, and of P, so far
      int both = 0;                                // tiles so far that both halves need
      bool ok = true;
      // Where both halves walk over the same keys they take turns, the first one first: left alone they fall into step, with
      // both at their exponentials and then both at the tensor cores.  A hint only: the wait is short and may be given up.
      auto take_turn = [&](bool first_of_tile) {
        for (int i = 0; i < 256; ++i)
          if (h == 0 ? first_of_tile || turns[1] >= both : turns[0] > both) break;
      };
      // Every slot is waited for and given back, also where this half needs nothing of it: a slot is free when both halves
      // have said so once.
      auto wait_slot = [&](int i) {
        return __all_sync(0xffffffffu, mbar_wait(full_bar(i % NS), (i / NS) & 1u, abort_flag)) != 0;
      };
      while (ok && w.next()) {
        const KeyTiles<kTile> tiles = tiles_of(), need = half_tiles(h), other = half_tiles(h ^ 1);
        const int n = tiles.count(), total = need.count();
        int issued = 0, nth = 0;
        auto scores = [&](int it) {                // S of tile `it`, whose K is there
          if (need.has(tile_at(tiles, it))) {
            ++issued;
            if (one) {
              const uint64_t kd = make_desc_kmajor_rows(ring + ((base + 2 * it) % NS) * TB, 128);
              const uint64_t qd = make_desc_kmajor_rows(q_base + h * TB, 128);
#pragma unroll
              for (int k = 0; k < DP / 16; ++k) {
                const uint64_t off = ((k >> 2) * (kTile * 128) + (k & 3) * 32) >> 4;  // the address field counts 16 bytes
                umma_bf16(t_s, qd + off, kd + off, idesc_s, k != 0);
              }
              umma_commit(s_bar(h));
              if (issued == total) umma_commit(q_empty_bar(h));
            }
          }
          if (one) umma_commit(empty_bar((base + 2 * it) % NS));
        };
        if (total > 0) {
          ok = __all_sync(0xffffffffu, mbar_wait(q_bar(h), q_used & 1u, abort_flag));
          ++q_used;
        }
        ok = ok && (n == 0 || wait_slot(base));
        tc_fence_after();
        if (ok && n > 0) scores(0);
        for (int it = 0; it < n && ok; ++it) {
          const int vi = base + 2 * it + 1;
          ok = (it + 1 >= n || wait_slot(vi + 1)) && wait_slot(vi);
          if (!ok) break;
          if (need.has(tile_at(tiles, it))) {
            const int j0 = tile_at(tiles, it) * kTile;
            const uint32_t vb = ring + (vi % NS) * TB;
            if (j0 + kTile > w.sq.lk) {
              // rows behind the last key belong to someone else and may hold anything; P is zero there, V has to be finite
              // (both halves' warps clear them, with the same zeros)
              const int first = w.sq.lk - j0;
              for (int i = lane; i < (kTile - first) * 8 * NB; i += 32) {
                const int c = i & 7, blk = (i >> 3) % NB, r = first + (i >> 3) / NB;
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vb + blk * (kTile * 128) + r * 128 + c * 16),
                             "r"(0)
                             : "memory");
              }
              fence_proxy_async_smem();
              __syncwarp();
            }
            // the first product of a tile overwrites O, which the tile before has to have been read out of
            if (nth == 0) ok = __all_sync(0xffffffffu, mbar_wait(o_empty_bar(h), q_used & 1u, abort_flag));
            const uint64_t vd = make_desc(vb, kTile * 128, 1024);
#pragma unroll
            for (int c = 0; c < 2; ++c) {                      // the two halves of P as they come
              ok = ok && __all_sync(0xffffffffu, mbar_wait(p_bar(h) + 16u * c, done & 1u, abort_flag));
              if (!ok) break;
              if (c == 0 && other.has(tile_at(tiles, it))) take_turn(nth == 0);
              tc_fence_after();
              if (one) {
#pragma unroll
                for (int k = 4 * c; k < 4 * c + 4; ++k)
                  umma_bf16_ts(t_o, t_s + k * 8, vd + k * (2048 >> 4), idesc_o, (nth | k) != 0);
                if (c == 0) umma_commit(v_bar(h));
              }
            }
            if (!ok) break;
            ++done;
            if (++nth == total && one) umma_commit(o_bar(h));
          }
          if (one) umma_commit(empty_bar(vi % NS));
          tc_fence_after();
          if (it + 1 < n) scores(it + 1);
          if (need.has(tile_at(tiles, it)) && other.has(tile_at(tiles, it))) {
            ++both;
            if (one) turns[h] = both;
          }
        }
        base += 2 * n;
      }
      if (!ok && lane == 0) {
        *abort_flag = 1;
        if (a.status) atomicExch(a.status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ---------------- softmax: one row per thread ----------------
    const int h = warp >> 2;
    const int row = h * kTile + (warp & 3) * 32 + lane;      // in the block
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lanes + h * kTile, o_addr = tmem + lanes + 2 * kTile + h * DP;
    // scores in base 2: exp2 of them is e^s
    const float mul = CAP ? a.scale / a.softcap : a.scale * kLog2e;
    const float cap2 = a.softcap * kLog2e;
    constexpr bool kTransformed = CAP || BIAS;               // else the factor goes into the exponent's multiply-add
    constexpr bool kGuessed = CAP && !BIAS;                  // m may start from 0
    const float to2 = kTransformed ? 1.f : mul;
    bool ok = true;
    int cnt = 0;                                             // tiles of this half so far, over all row tiles
    int o_used = 0;
    // Waits for its stores too: a tile may rescale O twice, and only that wait orders a load behind a store.
    auto scale_o = [&](float f) {
#pragma unroll 1
      for (int i = 0; i < DP / 16; ++i) {
        uint32_t o[16];
        tmem_ld16(o_addr + i * 16, o);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
        tmem_st16(o_addr + i * 16, o);
      }
      tmem_st_wait();
    };
    while (ok && w.next()) {
      const KeyTiles<kTile> tiles = tiles_of(), need = half_tiles(h);
      const int n = tiles.count(), total = need.count(), rows = rows_of();
      const int pos = w.sq.shift + w.row0 + row;
      const RowKeys keys = row_keys(w.sq, a.causal, a.window, pos);
      const float slope2 = BIAS ? a.slopes[w.head] * kLog2e : 0.f;
      // m in base 2; the sums of p as taken, for the log-sum-exp, and as rounded, by which O is divided: the weights that
      // the product uses then sum to one, and a row with one large weight keeps its value
      float m = kGuessed && cap2 <= 96.f ? 0.f : -INFINITY, l = 0.f, l_used = 0.f;
      float tile_sum = 0.f;                                    // the last tile's part of l
      int nth = 0;
      for (int it = 0; it < n && ok; ++it) {
        const int t = tile_at(tiles, it);
        if (!need.has(t)) continue;
        ok = __all_sync(0xffffffffu, mbar_wait(s_bar(h), cnt & 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        // S is there, so the products before it have finished and O stands still
        if (__any_sync(0xffffffffu, tile_sum > kRaise)) {      // the last tile's p had grown: m follows
          const float k = tile_sum > kRaise ? ceilf(log2f(tile_sum)) : 0.f, f = ex2(-k);
          m += k;
          l *= f;
          l_used *= f;
          scale_o(f);
        }
        tile_sum = 0.f;
#pragma unroll 1
        for (int c = 0; c < 2 && ok; ++c) {
          const int j0 = t * kTile + c * 64;
          // what the warp's rows see of these keys: all, some (then hidden scores become -inf), or nothing
          const int lo = keys.lo - j0, hi = keys.hi - j0, pre = keys.prefix - j0;
          const bool whole = __all_sync(0xffffffffu, (lo <= 0 && hi >= 64) || pre >= 64);
          if (__all_sync(0xffffffffu, min(hi, 64) <= max(lo, 0) && pre <= 0)) {
            uint32_t zero[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) zero[i] = 0;
            tmem_st32(s_addr + c * 32, zero);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_bar(h) + 16u * c);
            continue;
          }
          float x[64];
          tmem_ld32(s_addr + c * 64, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
          tmem_ld32(s_addr + c * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
          tmem_ld_wait();
          if (CAP) {
            tanh_all(x, mul);
#pragma unroll
            for (int j = 0; j < 64; j += 2) unpair2(mul2(pair2(x[j], x[j + 1]), pair2(cap2, cap2)), x[j], x[j + 1]);
          }
          if (BIAS) {
            const float d = (float)(pos - j0);
#pragma unroll
            for (int j = 0; j < 64; ++j) x[j] = fmaf(-slope2, fabsf(d - (float)j), CAP ? x[j] : x[j] * mul);
          }
          if (!whole) {                                        // a bit and a selection a score, whatever the mask
#pragma unroll
            for (int b = 0; b < 64; b += 32) {
              const uint32_t seen = seen_bits(lo - b, hi - b, pre - b);
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(seen & (1u << j))) x[b + j] = -INFINITY;
            }
          }
          uint32_t pk[32];
          float sum, sum_used;
          bool reset = m == -INFINITY;                         // nothing seen yet; below: p far from one
#pragma unroll 1
          for (int attempt = 0; attempt < 2; ++attempt) {      // over their own maximum p are at most about 1
            if (__any_sync(0xffffffffu, reset)) {
              float mx[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
              for (int j = 4; j < 64; ++j) mx[j & 3] = fmaxf(mx[j & 3], x[j]);
              const float mt = ceilf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * to2);
              const bool none = kGuessed ? l == 0.f : m == -INFINITY;   // nothing seen before: l and O are zero
              const float m_new = !reset ? m : kGuessed && none ? mt : fmaxf(mt, m);
              const float f = none ? 0.f : ex2(m - m_new);
              m = m_new;
              l *= f;
              l_used *= f;
              tile_sum *= f;
              if (c == 1) {                                    // the first half's P may still be on its way into O
                ok = __all_sync(0xffffffffu, mbar_wait(v_bar(h), cnt & 1u, abort_flag));
                if (!ok) break;
                tc_fence_after();
              }
              if (nth > 0 || c == 1) scale_o(f);
            }
            const float shift = m == -INFINITY ? 0.f : -m;
            const uint64_t mul_2 = pair2(to2, to2), shift_2 = pair2(shift, shift);
            uint64_t acc[2] = {0ull, 0ull}, used[2] = {0ull, 0ull};
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              uint64_t v = pair2(x[2 * i], x[2 * i + 1]);
              v = kTransformed ? add2(v, shift_2) : fma2(v, mul_2, shift_2);
              float e0, e1;
              unpair2(v, e0, e1);
              e0 = ex2(e0);
              e1 = ex2(e1);
              acc[i & 1] = add2(acc[i & 1], pair2(e0, e1));
              pk[i] = bf16x2(e0, e1);
              used[i & 1] = add2(used[i & 1], pair2(bf16_lo(pk[i]), bf16_hi(pk[i])));
            }
            float l0, l1;
            unpair2(add2(acc[0], acc[1]), l0, l1);
            sum = l0 + l1;
            unpair2(add2(used[0], used[1]), l0, l1);
            sum_used = l0 + l1;
            tmem_st32(s_addr + c * 32, pk);                    // over scores of the tile's first half
            reset = sum > kRetake || (kGuessed && l == 0.f && sum > 0.f && sum < 1.f / kRetake);
            if (!__any_sync(0xffffffffu, reset)) break;
            tmem_st_wait();                                    // the next attempt writes the same columns
          }
          if (!ok) break;
          l += sum;
          l_used += sum_used;
          tile_sum += sum;
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_bar(h) + 16u * c);
        }
        ++cnt;
        ++nth;
      }
      if (ok && total > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(o_bar(h), o_used & 1u, abort_flag));
        ++o_used;
        tc_fence_after();
      }
      if (ok && rows > h * kTile) {
        const float inv = l > 0.f || l != l ? 1.f / l_used : 0.f;   // a row that sees nothing gives zeros
        const bool mine = row < rows;
        bf16* dst = reinterpret_cast<bf16*>(a.out) + (size_t)(w.sq.q0 + w.row0 + (mine ? row : 0)) * a.o_stride +
                    (size_t)w.head * a.head_dim;
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) {
          uint32_t o[32];
          if (total > 0) {
            tmem_ld32(o_addr + c * 32, o);
            tmem_ld_wait();
            if (c == DP / 32 - 1) {                            // O may be written again
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(o_empty_bar(h));
            }
          }
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            if (mine && c * 32 + g * 8 < a.head_dim) {
              uint4 v = make_uint4(0, 0, 0, 0);
              if (total > 0) {
                uint32_t* vp = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  vp[i] = bf16x2(__uint_as_float(o[g * 8 + 2 * i]) * inv, __uint_as_float(o[g * 8 + 2 * i + 1]) * inv);
              }
              *reinterpret_cast<uint4*>(dst + c * 32 + g * 8) = v;
            }
          }
        }
        if (a.lse && mine)
          a.lse[(size_t)w.head * a.q_rows + w.sq.q0 + w.row0 + row] = (m + log2f(l)) * kLn2;
      }
    }
    if (!ok && lane == 0) {
      *abort_flag = 1;
      if (a.status) atomicExch(a.status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    for (int i = 0; i < 200; ++i) __nanosleep(5000);         // let copies that may still be in flight land
  }
  tc_fence_after();
  if (warp == kMmaWarp) {
    __syncwarp();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <int DP, bool CAP, bool BIAS>
cudaError_t launch(const FwdParams& p, unsigned grid, cudaStream_t st) {
  static bool done[64];
  cudaError_t e = allow_smem(attn_fwd_tc_kernel<DP, CAP, BIAS>, kSmemBytes<DP>, done);
  if (e != cudaSuccess) return e;
  return launch_behind(attn_fwd_tc_kernel<DP, CAP, BIAS>, grid, kThreads, kSmemBytes<DP>, st, p);
}

template <int DP>
cudaError_t launch_dp(const FwdParams& p, unsigned grid, cudaStream_t st) {
  if (p.a.softcap > 0.f) return p.a.slopes ? launch<DP, true, true>(p, grid, st) : launch<DP, true, false>(p, grid, st);
  return p.a.slopes ? launch<DP, false, true>(p, grid, st) : launch<DP, false, false>(p, grid, st);
}

}  // namespace

cudaError_t launch_attn_forward_tc(const AttnArgs& a, cudaStream_t st) {
  FwdParams p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  const long long kr = a.k_rows > 0 ? a.k_rows : 1;          // without keys no tile is loaded
  if (!tc_encode_heads(&p.q_map, a.q, a.q_rows, a.q_heads, a.head_dim, a.q_stride, kTile) ||
      !tc_encode_heads(&p.k_map, a.k, kr, a.kv_heads, a.head_dim, a.k_stride, kTile) ||
      !tc_encode_heads(&p.v_map, a.v, kr, a.kv_heads, a.head_dim, a.v_stride, kTile))
    return cudaErrorInvalidValue;
  const long long most = ((long long)(a.q_rows + kFwdTile - 1) / kFwdTile + a.n_seqs) * a.q_heads;
  if (most > 0x7fff0000LL) return cudaErrorInvalidValue;
  const int sms = attn_sm_count();
  const long long grid = most < sms ? most : sms;            // one block per SM, which walks over the tiles
  return a.head_dim <= 64 ? launch_dp<64>(p, (unsigned)grid, st) : launch_dp<128>(p, (unsigned)grid, st);
}

}  // namespace mixlora
