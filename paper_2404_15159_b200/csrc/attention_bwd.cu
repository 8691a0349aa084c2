// Masked attention, backward, bf16, on the tensor cores.
//
//   p_ij  = e^(s_ij - lse_i)                       from the forward's log-sum-exp
//   dv_j  = sum_i p_ij do_i
//   ds_ij = p_ij (do_i . v_j - delta_i) c'_ij      delta_i = do_i . o_i;  c' = 1 - tanh^2 of a capped score, else 1
//   dq_i  = scale sum_j ds_ij k_j                  dk_j = scale sum_i ds_ij q_i
//
// Two launches over the same tiles: one owns 128 keys and walks over the query rows that see them (and over the query
// heads that share the key head) for dk and dv, one owns 128 query rows and walks over their keys for dq.  Scores and
// p are formed in both: seven products of a tile instead of five, but every gradient is summed by one block in one
// order, in TMEM, without atomics.  p and ds are rounded to bf16 for their products (half a step, 2^-8, of a value that
// is summed over many), everything else is fp32.
//
// A tile of dk / dv is 2048 cycles of the tensor pipe at 128 values a head and takes about 3100, one of dq 1536 and about
// 2200: what is left over is the chain from a product to the elements and back.  Measured: 8192 rows in 4 documents, 32 / 8
// heads of 128, causal: delta 32 us, dk and dv 304 us, dq 250 us (0.87 PFLOP/s of the seven products).
#include <cuda.h>
#include <string.h>

#include "attention.cuh"
#include "tc_ptx.cuh"

namespace mixlora {
namespace {
using namespace tc;

constexpr int kTile = 128;
constexpr int kThreads = 384;                    // two groups of 4 warps on the elements, a load warp, an MMA warp
// A block starts with 168 registers a thread (384 x 168 = 64512); the element groups take 208 and the third group keeps 88:
// (2 x 208 + 88) x 128 = 64512.
constexpr int kLoadWarp = 8, kMmaWarp = 9;
constexpr int kTmemCols = 512;
constexpr int kRowWarp = 10;                     // of the key kernel: carries lse and delta
// The walked tiles come in two streams.  Stream A (q; of the query kernel: k) is read by a tile's first and last product,
// stream B (do; v) is done earlier: three and two stages, which is what shared memory holds at 128 values a head.
constexpr int kStagesA = 3, kStagesB = 2;
template <int DP> constexpr uint32_t kTileBytes = kTile * DP * 2;
constexpr uint32_t kRowBytes = 2 * kTile * 4;    // minus lse and minus delta of a query tile, two stages
template <int DP> constexpr uint32_t kSmemBytes = (2 + kStagesA + kStagesB) * kTileBytes<DP> + 2 * kRowBytes + 256;

struct BwdParams {
  AttnArgs a;
  CUtensorMap q_map, k_map, v_map, do_map;
};

struct Ctl {
  uint32_t bars;
  volatile int* abort_flag;
  __device__ __forceinline__ uint32_t full_a(int i) const { return bars + 8u * (i % kStagesA); }
  __device__ __forceinline__ uint32_t empty_a(int i) const { return bars + 8u * (kStagesA + i % kStagesA); }
  __device__ __forceinline__ uint32_t full_b(int i) const { return bars + 8u * (2 * kStagesA + i % kStagesB); }
  __device__ __forceinline__ uint32_t empty_b(int i) const { return bars + 8u * (2 * kStagesA + kStagesB + i % kStagesB); }
  __device__ __forceinline__ uint32_t at(int k) const { return bars + 8u * (2 * kStagesA + 2 * kStagesB + k); }
  __device__ __forceinline__ uint32_t own() const { return at(0); }                      // the block's own tiles
  __device__ __forceinline__ uint32_t s(int k) const { return at(1 + k); }               // scores are there
  __device__ __forceinline__ uint32_t dp() const { return at(3); }                       // do . v is there
  __device__ __forceinline__ uint32_t p() const { return at(4); }                        // p is written
  __device__ __forceinline__ uint32_t ds() const { return at(5); }                       // ds is written
  __device__ __forceinline__ uint32_t acc() const { return at(6); }                      // the sums are final
  __device__ __forceinline__ uint32_t rows_full(int i) const { return at(7 + (i & 1)); }
  __device__ __forceinline__ uint32_t rows_empty(int i) const { return at(9 + (i & 1)); }
  __device__ __forceinline__ uint32_t own_empty() const { return at(11); }               // the own tiles have been used
  __device__ __forceinline__ uint32_t acc_empty() const { return at(12); }               // the sums have been read
  // waits for use number i / stages of a stage
  __device__ __forceinline__ bool wait_full_a(int i) const { return mbar_wait(full_a(i), (i / kStagesA) & 1u, abort_flag); }
  __device__ __forceinline__ bool wait_empty_a(int i) const { return mbar_wait(empty_a(i), ((i / kStagesA) & 1u) ^ 1u, abort_flag); }
  __device__ __forceinline__ bool wait_full_b(int i) const { return mbar_wait(full_b(i), (i / kStagesB) & 1u, abort_flag); }
  __device__ __forceinline__ bool wait_empty_b(int i) const { return mbar_wait(empty_b(i), ((i / kStagesB) & 1u) ^ 1u, abort_flag); }
};
constexpr int kBars = 2 * kStagesA + 2 * kStagesB + 13;

template <int DP>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int row) {
#pragma unroll
  for (int j = 0; j < DP / 64; ++j) tma_load_3d(dst + j * (kTile * 128), map, bar, j * 64, head, row);
}
// Rows [first, 128) of a tile belong to someone else and may hold anything; as the summed index of a product, and as the
// columns of scores and dP, they have to be finite (p and ds are zero there).  One warp.
template <int DP>
__device__ __forceinline__ void clear_rows(uint32_t tile, int first) {
  constexpr int NB = DP / 64;
  for (int i = threadIdx.x & 31; i < (kTile - first) * 8 * NB; i += 32) {
    const int c = i & 7, blk = (i >> 3) % NB, r = first + (i >> 3) / NB;
    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + blk * (kTile * 128) + r * 128 + c * 16), "r"(0)
                 : "memory");
  }
}
// D[128 x 128] = A B^T over the head's `dim` values, both tiles K-major.  Here and below a head of 80 or 96 in tiles of 128
// is multiplied as what it is (dk/dv 53 to 51 us, dq 38 to 36 at 2901 rows, window 500, 20 heads of 80; in the forward
// kernel the check costs a head of 128 1 % and gains one of 80 as little, so that one multiplies the zeros).
template <int DP>
__device__ __forceinline__ void issue_nt(uint32_t d, uint32_t a, uint32_t b, int dim) {
  const uint32_t idesc = make_idesc(kTile, 0, 0);
  const uint64_t ad = make_desc_kmajor_rows(a, 128), bd = make_desc_kmajor_rows(b, 128);
#pragma unroll
  for (int k = 0; k < DP / 16; ++k) {
    const uint64_t off = ((k >> 2) * (kTile * 128) + (k & 3) * 32) >> 4;          // the address field counts 16 bytes
    if (k * 16 < dim) umma_bf16(d, ad + off, bd + off, idesc, k != 0);
  }
}
// D[128 x dim] += A B, A bf16 [128 x 128] in TMEM (columns 0-31 and 64-95 of its region), B rows = the summed index
template <int DP>
__device__ __forceinline__ void issue_ts(uint32_t d, uint32_t a, uint32_t b, bool accumulate, int dim) {
  const uint32_t idesc = make_idesc((dim + 15) / 16 * 16, 0, 1);
  const uint64_t bd = make_desc(b, kTile * 128, 1024);
#pragma unroll
  for (int k = 0; k < kTile / 16; ++k)
    umma_bf16_ts(d, a + (k >> 2) * 64 + (k & 3) * 8, bd + k * (2048 >> 4), idesc, accumulate || k != 0);
}
// 64 zeros of p or ds
__device__ __forceinline__ void store_zeros(uint32_t addr) {
  uint32_t z[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0;
  tmem_st16(addr, z);
  tmem_st16(addr + 16, z);
}
// N values of a row of the sums to memory, those before `valid` (zeros where there are no sums); `empty` is told once
// they have been read.
template <int N>
__device__ __forceinline__ void store_row(uint32_t acc, bool any, uint32_t empty, float mul, bool mine, bf16* dst,
                                          int valid) {
#pragma unroll
  for (int c = 0; c < N / 32; ++c) {
    uint32_t v[32];
    if (any) {
      tmem_ld32(acc + c * 32, v);
      tmem_ld_wait();
      if (c == N / 32 - 1) {
        tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(empty);
      }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g)
      if (mine && c * 32 + g * 8 < valid) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (any) {
          uint32_t* wp = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            wp[i] = bf16x2(__uint_as_float(v[g * 8 + 2 * i]) * mul, __uint_as_float(v[g * 8 + 2 * i + 1]) * mul);
        }
        *reinterpret_cast<uint4*>(dst + c * 32 + g * 8) = w;
      }
  }
}

// Block setup shared by both kernels: barriers and TMEM, whose address is returned.  `readers`: warps that read the sums.
__device__ __forceinline__ uint32_t block_begin(const Ctl& c, uint32_t* slot, int readers) {
  if (threadIdx.x == 32) {
    for (int i = 0; i < kStagesA; ++i) { mbar_init(c.full_a(i), 1); mbar_init(c.empty_a(i), 1); }
    for (int i = 0; i < kStagesB; ++i) { mbar_init(c.full_b(i), 1); mbar_init(c.empty_b(i), 1); }
    mbar_init(c.own(), 1); mbar_init(c.s(0), 1); mbar_init(c.s(1), 1); mbar_init(c.dp(), 1); mbar_init(c.acc(), 1);
    mbar_init(c.p(), 8); mbar_init(c.ds(), 8);
    for (int i = 0; i < 2; ++i) { mbar_init(c.rows_full(i), 1); mbar_init(c.rows_empty(i), 8); }
    mbar_init(c.own_empty(), 1); mbar_init(c.acc_empty(), readers);
    *c.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if ((threadIdx.x >> 5) == kMmaWarp) {
    tmem_alloc(smem_u32(slot), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  return warp_uniform(*slot);
}
__device__ __forceinline__ void give_up(const Ctl& c, int32_t* status) {
  *c.abort_flag = 1;
  if (status) atomicExch(status, (int)MIXLORA_ERR_DEVICE_TIMEOUT);
}
__device__ __forceinline__ void block_end(const Ctl& c, uint32_t tmem) {
  tc_fence_before();
  __syncthreads();
  if (*c.abort_flag) {
    for (int i = 0; i < 200; ++i) __nanosleep(5000);         // let copies that may still be in flight land
  }
  tc_fence_after();
  if ((threadIdx.x >> 5) == kMmaWarp) {
    __syncwarp();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// p of two neighbouring scores: 2^(score - log-sum-exp), in base 2; with a cap the scores are tanh already, and the slope
// comes back too.  `neg_lse` is minus the log-sum-exp, `d0`, `d1` are the distances.
template <bool CAP, bool BIAS>
struct Score {
  float mul, factor, slope2;
  __device__ __forceinline__ Score(const AttnArgs& a, int head)
      : mul(a.scale / a.softcap), factor(CAP ? a.softcap * kLog2e : a.scale * kLog2e),
        slope2(BIAS ? a.slopes[head] * kLog2e : 0.f) {}
  template <int N>
  __device__ __forceinline__ void cap(float (&s)[N]) const {
    if (CAP) tanh_all(s, mul);
  }
  __device__ __forceinline__ void probs(float s0, float s1, uint64_t neg_lse, float d0, float d1, float& p0, float& p1,
                                        uint64_t& cap_slope) const {
    const uint64_t s = pair2(s0, s1);
    if (CAP) cap_slope = fma2(pair2(-s0, -s1), s, pair2(1.f, 1.f));
    const uint64_t x = fma2(s, pair2(factor, factor), neg_lse);
    float x0, x1;
    unpair2(x, x0, x1);
    if (BIAS) {
      x0 = fmaf(-slope2, fabsf(d0), x0);
      x1 = fmaf(-slope2, fabsf(d1), x1);
    }
    p0 = ex2(x0);
    p1 = ex2(x1);
  }
};

// dk, dv of 128 keys of a key head.  TMEM: S^T and dP^T [128 keys x 128 rows] (p^T and ds^T are written over them as
// bf16 and read from there by the products), dv, dk.  While the element groups work on p the tensor cores form the
// next dP^T and dk, while they work on ds the next S^T and dv.
template <int DP, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) attn_bwd_kv_kernel(const __grid_constant__ BwdParams p) {
  constexpr uint32_t TB = kTileBytes<DP>;
  extern __shared__ __align__(1024) uint8_t smem[];          // the swizzle counts from 1024-byte boundaries
  const uint32_t k_tile = smem_u32(smem), v_tile = k_tile + TB;
  auto q_at = [&](int i) { return k_tile + (2 + i % kStagesA) * TB; };
  auto do_at = [&](int i) { return k_tile + (2 + kStagesA + i % kStagesB) * TB; };
  float* rows_smem = reinterpret_cast<float*>(smem + (2 + kStagesA + kStagesB) * TB);
  uint8_t* ctl = reinterpret_cast<uint8_t*>(rows_smem) + 2 * kRowBytes;
  uint32_t* slot = reinterpret_cast<uint32_t*>(ctl + 8 * kBars);
  const Ctl c{smem_u32(ctl), reinterpret_cast<volatile int*>(slot + 1)};
  const AttnArgs& a = p.a;
  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t tmem = block_begin(c, slot, 8);
  const uint32_t t_s = tmem, t_dp = tmem + kTile, t_dv = tmem + 2 * kTile, t_dk = t_dv + DP;
  let_next_start();
  wait_for_last();                               // the plan, and delta
  TileWalk w(a.k_tiles, a.n_k_tiles, a.kv_heads);            // w.head is the key head
  // of the tile at hand: the query tiles of a head that see it, from row `lo`, and the steps over all heads that share it
  int lo = 0, per_head = 0;
  auto steps = [&] {
    int hi;
    query_rows(w.sq, a.causal, a.window, w.row0, min(w.row0 + kTile, w.sq.lk), &lo, &hi);
    lo = lo / kTile * kTile;
    per_head = hi > lo ? (hi - lo + kTile - 1) / kTile : 0;
    return per_head * a.group;
  };
  auto head_of = [&](int i) { return w.head * a.group + i / per_head; };
  auto row_of = [&](int i) { return lo + (i % per_head) * kTile; };

  // In every role `at` counts the steps of the tiles before: stages and barrier phases go on from tile to tile.
  if (warp >= kLoadWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kLoadWarp) {
      if (lane == 0) {
        bool ok = true;
        int at = 0, used = 0;                                  // used: tiles whose keys have been loaded
        while (ok && w.next()) {
          const int n = steps();
          if (n == 0) continue;
          if (!mbar_wait(c.own_empty(), (used & 1u) ^ 1u, c.abort_flag)) { ok = false; break; }
          ++used;
          mbar_expect_tx(c.own(), 2 * TB);
          load_tile<DP>(k_tile, &p.k_map, c.own(), w.head, w.sq.k0 + w.row0);
          load_tile<DP>(v_tile, &p.v_map, c.own(), w.head, w.sq.k0 + w.row0);
          for (int i = 0; i < n; ++i, ++at) {
            if (!c.wait_empty_a(at)) { ok = false; break; }
            mbar_expect_tx(c.full_a(at), TB);
            load_tile<DP>(q_at(at), &p.q_map, c.full_a(at), head_of(i), w.sq.q0 + row_of(i));
            if (!c.wait_empty_b(at)) { ok = false; break; }
            mbar_expect_tx(c.full_b(at), TB);
            load_tile<DP>(do_at(at), &p.do_map, c.full_b(at), head_of(i), w.sq.q0 + row_of(i));
          }
        }
        if (!ok) give_up(c, a.status);
      }
    } else if (warp == kRowWarp) {
      bool ok = true;
      int at = 0;
      while (ok && w.next()) {
        const int n = steps();
        for (int i = 0; i < n; ++i, ++at) {
          float v[2][kTile / 32];
          const size_t first = (size_t)head_of(i) * a.q_rows + w.sq.q0 + row_of(i);
#pragma unroll
          for (int x = 0; x < kTile / 32; ++x) {
            const bool on = row_of(i) + x * 32 + lane < w.sq.lq;
            v[0][x] = on ? -a.lse2[first + x * 32 + lane] : -INFINITY;
            v[1][x] = on ? -a.delta[first + x * 32 + lane] : 0.f;
          }
          ok = __all_sync(0xffffffffu, mbar_wait(c.rows_empty(at), ((at >> 1) & 1u) ^ 1u, c.abort_flag));
          if (!ok) break;
          float* dst = rows_smem + (at & 1) * (2 * kTile) + lane;
#pragma unroll
          for (int x = 0; x < kTile / 32; ++x) {
            dst[x * 32] = v[0][x];
            dst[kTile + x * 32] = v[1][x];
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(c.rows_full(at));
        }
      }
      if (!ok && lane == 0) give_up(c, a.status);
    } else if (warp == kMmaWarp) {
      const bool one = elect_one();
      bool ok = true;
      int at = 0, used = 0;
      // a stream's tile i is in shared memory, its rows behind the last cleared
      auto tail = [&](int i, uint32_t tile) {
        const int valid = w.sq.lq - row_of(i);
        if (valid < kTile) {
          clear_rows<DP>(tile, valid);
          fence_proxy_async_smem();
          __syncwarp();
        }
        tc_fence_after();
      };
      auto scores = [&](int i) {
        if (!__all_sync(0xffffffffu, c.wait_full_a(at + i))) return false;
        tail(i, q_at(at + i));
        if (one) {
          issue_nt<DP>(t_s, k_tile, q_at(at + i), a.head_dim);
          umma_commit(c.s(0));
        }
        return true;
      };
      auto grads = [&](int i) {
        if (!__all_sync(0xffffffffu, c.wait_full_b(at + i))) return false;
        tail(i, do_at(at + i));
        if (one) {
          issue_nt<DP>(t_dp, v_tile, do_at(at + i), a.head_dim);
          umma_commit(c.dp());
        }
        return true;
      };
      while (ok && w.next()) {
        const int n = steps();
        if (n == 0) continue;
        ok = __all_sync(0xffffffffu, mbar_wait(c.own(), used & 1u, c.abort_flag)) && scores(0) && grads(0) &&
             __all_sync(0xffffffffu, mbar_wait(c.acc_empty(), (used & 1u) ^ 1u, c.abort_flag));
        ++used;
        for (int i = 0; i < n && ok; ++i) {
          ok = __all_sync(0xffffffffu, mbar_wait(c.p(), (at + i) & 1u, c.abort_flag));
          if (!ok) break;
          tc_fence_after();
          if (one) {
            issue_ts<DP>(t_dv, t_s, do_at(at + i), i > 0, a.head_dim);
            umma_commit(c.empty_b(at + i));
          }
          ok = i + 1 >= n || scores(i + 1);
          ok = ok && __all_sync(0xffffffffu, mbar_wait(c.ds(), (at + i) & 1u, c.abort_flag));
          if (!ok) break;
          tc_fence_after();
          if (one) {
            issue_ts<DP>(t_dk, t_dp, q_at(at + i), i > 0, a.head_dim);
            umma_commit(c.empty_a(at + i));
            if (i + 1 == n) { umma_commit(c.acc()); umma_commit(c.own_empty()); }
          }
          ok = i + 1 >= n || grads(i + 1);
        }
        at += n;
      }
      if (!ok && lane == 0) give_up(c, a.status);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ---------------- elements: one key per thread, half of the tile's rows per group ----------------
    const int half = warp >> 2, key = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = t_s + lanes + half * 64, dp_addr = t_dp + lanes + half * 64;
    bool ok = true;
    int at = 0, used = 0;
    while (ok && w.next()) {
      const int n = steps(), j0 = w.row0, j = j0 + key, keys = min(kTile, w.sq.lk - j0);
      for (int i = 0; i < n && ok; ++i, ++at) {
        const int i0 = row_of(i) + half * 64;
        const Score<CAP, BIAS> score(a, head_of(i));
        const float* neg_lse = rows_smem + (at & 1) * (2 * kTile) + half * 64;
        const float* neg_delta = neg_lse + kTile;
        const int pos0 = w.sq.shift + i0;
        // the rows of these 64 that see this key: [r_lo, r_hi); what that comes to for the warp's keys: all, some (hidden
        // ones become zeros), or nothing
        int r_lo = 0, r_hi = 0;
        if (j < w.sq.lk) query_rows(w.sq, a.causal, a.window, j, j + 1, &r_lo, &r_hi);
        r_lo -= i0;
        r_hi -= i0;
        const bool whole = __all_sync(0xffffffffu, r_lo <= 0 && r_hi >= 64);
        const bool none = __all_sync(0xffffffffu, min(r_hi, 64) <= max(r_lo, 0));
        ok = __all_sync(0xffffffffu, mbar_wait(c.rows_full(at), (at >> 1) & 1u, c.abort_flag) &&
                                         mbar_wait(c.s(0), at & 1u, c.abort_flag));
        if (!ok) break;
        tc_fence_after();
        float pr[2][32];
        if (none) {
          store_zeros(s_addr);
        } else {
          const float d = (float)(pos0 - j);
#pragma unroll
          for (int c0 = 0; c0 < 2; ++c0) {
            uint64_t cs[CAP ? 16 : 1];
            float (&pc)[32] = pr[c0];
            tmem_ld32(s_addr + c0 * 32, *reinterpret_cast<uint32_t(*)[32]>(&pc[0]));
            tmem_ld_wait();
            score.cap(pc);
#pragma unroll
            for (int x = 0; x < 32; x += 4) {
              const float4 ls = *reinterpret_cast<const float4*>(neg_lse + c0 * 32 + x);
              const float d0 = d + (float)(c0 * 32 + x);
              uint64_t& cs0 = cs[CAP ? x / 2 : 0];
              uint64_t& cs1 = cs[CAP ? x / 2 + 1 : 0];
              score.probs(pc[x], pc[x + 1], pair2(ls.x, ls.y), d0, d0 + 1.f, pc[x], pc[x + 1], cs0);
              score.probs(pc[x + 2], pc[x + 3], pair2(ls.z, ls.w), d0 + 2.f, d0 + 3.f, pc[x + 2], pc[x + 3], cs1);
            }
            if (!whole) {
              const uint32_t seen = seen_bits(r_lo - c0 * 32, r_hi - c0 * 32, 0);
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if (!(seen & (1u << x))) pc[x] = 0.f;
            }
            uint32_t pk[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) pk[x] = bf16x2(pc[2 * x], pc[2 * x + 1]);
            tmem_st16(s_addr + c0 * 16, pk);
            if (CAP) {                                           // from here on p times the cap's slope
#pragma unroll
              for (int x = 0; x < 32; x += 2) {
                float f0, f1;
                unpair2(mul2(pair2(pc[x], pc[x + 1]), cs[x / 2]), f0, f1);
                pc[x] = f0;
                pc[x + 1] = f1;
              }
            }
          }
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(c.p());
        ok = __all_sync(0xffffffffu, mbar_wait(c.dp(), at & 1u, c.abort_flag));
        if (!ok) break;
        tc_fence_after();
        if (none) {
          store_zeros(dp_addr);
        } else {
#pragma unroll
          for (int c0 = 0; c0 < 2; ++c0) {
            float dp[32];
            tmem_ld32(dp_addr + c0 * 32, *reinterpret_cast<uint32_t(*)[32]>(&dp[0]));
            tmem_ld_wait();
            uint32_t pk[16];
#pragma unroll
            for (int x = 0; x < 32; x += 4) {
              const float4 dl = *reinterpret_cast<const float4*>(neg_delta + c0 * 32 + x);
              const float* pv = pr[c0] + x;
              uint64_t u = add2(pair2(dp[x], dp[x + 1]), pair2(dl.x, dl.y)), v = add2(pair2(dp[x + 2], dp[x + 3]), pair2(dl.z, dl.w));
              u = mul2(u, pair2(pv[0], pv[1]));
              v = mul2(v, pair2(pv[2], pv[3]));
              float f0, f1, f2, f3;
              unpair2(u, f0, f1);
              unpair2(v, f2, f3);
              pk[x / 2] = bf16x2(f0, f1);
              pk[x / 2 + 1] = bf16x2(f2, f3);
            }
            tmem_st16(dp_addr + c0 * 16, pk);
          }
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) { mbar_arrive(c.ds()); mbar_arrive(c.rows_empty(at)); }
      }
      if (ok && n > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(c.acc(), used & 1u, c.abort_flag));
        ++used;
        tc_fence_after();
      }
      if (ok) {
        const bool mine = key < keys;
        const size_t row = (size_t)(w.sq.k0 + (mine ? j : 0));
        if (half == 0)
          store_row<DP>(t_dv + lanes, n > 0, c.acc_empty(), 1.f, mine,
                        reinterpret_cast<bf16*>(a.dv) + row * a.v_stride + (size_t)w.head * a.head_dim, a.head_dim);
        else
          store_row<DP>(t_dk + lanes, n > 0, c.acc_empty(), a.scale, mine,
                        reinterpret_cast<bf16*>(a.dk) + row * a.k_stride + (size_t)w.head * a.head_dim, a.head_dim);
      }
    }
    if (!ok && lane == 0) give_up(c, a.status);
  }
  block_end(c, tmem);
}

// dq of 128 rows of a head.  TMEM: two S tiles in turn (ds is written over the one it comes from), dP, dq.  The next S
// runs while the element groups work on this one, and the next dP as soon as this one has been read.
template <int DP, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) attn_bwd_q_kernel(const __grid_constant__ BwdParams p) {
  constexpr uint32_t TB = kTileBytes<DP>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t q_tile = smem_u32(smem), do_tile = q_tile + TB;
  auto k_at = [&](int i) { return q_tile + (2 + i % kStagesA) * TB; };
  auto v_at = [&](int i) { return q_tile + (2 + kStagesA + i % kStagesB) * TB; };
  uint8_t* ctl = smem + (2 + kStagesA + kStagesB) * TB + 2 * kRowBytes;
  uint32_t* slot = reinterpret_cast<uint32_t*>(ctl + 8 * kBars);
  const Ctl c{smem_u32(ctl), reinterpret_cast<volatile int*>(slot + 1)};
  const AttnArgs& a = p.a;
  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t tmem = block_begin(c, slot, 4);
  const uint32_t t_dp = tmem + 2 * kTile, t_dq = tmem + 3 * kTile;
  wait_for_last();
  TileWalk w(a.q_tiles, a.n_q_tiles, a.q_heads);
  auto rows_of = [&] { return min(kTile, w.sq.lq - w.row0); };
  auto tiles_of = [&] {
    const int p0 = w.sq.shift + w.row0;
    return key_tiles<kTile>(w.sq, a.causal, a.window, p0, p0 + rows_of() - 1);
  };

  if (warp >= kLoadWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kLoadWarp) {
      if (lane == 0) {
        bool ok = true;
        int at = 0, used = 0;
        while (ok && w.next()) {
          const KeyTiles<kTile> tiles = tiles_of();
          const int n = tiles.count(), kvh = w.head / a.group;
          if (n == 0) continue;
          if (!mbar_wait(c.own_empty(), (used & 1u) ^ 1u, c.abort_flag)) { ok = false; break; }
          ++used;
          mbar_expect_tx(c.own(), 2 * TB);
          load_tile<DP>(q_tile, &p.q_map, c.own(), w.head, w.sq.q0 + w.row0);
          load_tile<DP>(do_tile, &p.do_map, c.own(), w.head, w.sq.q0 + w.row0);
          for (int i = 0; i < n; ++i, ++at) {
            if (!c.wait_empty_a(at)) { ok = false; break; }
            mbar_expect_tx(c.full_a(at), TB);
            load_tile<DP>(k_at(at), &p.k_map, c.full_a(at), kvh, w.sq.k0 + tiles.at(i) * kTile);
            if (!c.wait_empty_b(at)) { ok = false; break; }
            mbar_expect_tx(c.full_b(at), TB);
            load_tile<DP>(v_at(at), &p.v_map, c.full_b(at), kvh, w.sq.k0 + tiles.at(i) * kTile);
          }
        }
        if (!ok) give_up(c, a.status);
      }
    } else if (warp == kMmaWarp) {
      const bool one = elect_one();
      bool ok = true;
      int at = 0, used = 0;
      KeyTiles<kTile> tiles;
      // a stream's tile i is in shared memory, its keys behind the last cleared
      auto tail = [&](int i, uint32_t tile) {
        const int valid = w.sq.lk - tiles.at(i) * kTile;
        if (valid < kTile) {
          clear_rows<DP>(tile, valid);
          fence_proxy_async_smem();
          __syncwarp();
        }
        tc_fence_after();
      };
      auto scores = [&](int i) {                               // over ds of two tiles ago, which its product has read
        if (!__all_sync(0xffffffffu, c.wait_full_a(at + i))) return false;
        tail(i, k_at(at + i));
        if (one) {
          issue_nt<DP>(tmem + ((at + i) & 1) * kTile, q_tile, k_at(at + i), a.head_dim);
          umma_commit(c.s((at + i) & 1));
        }
        return true;
      };
      auto grads = [&](int i) {
        if (!__all_sync(0xffffffffu, c.wait_full_b(at + i))) return false;
        tail(i, v_at(at + i));
        if (one) {
          issue_nt<DP>(t_dp, do_tile, v_at(at + i), a.head_dim);
          umma_commit(c.dp());
          umma_commit(c.empty_b(at + i));
        }
        return true;
      };
      while (ok && w.next()) {
        tiles = tiles_of();
        const int n = tiles.count();
        if (n == 0) continue;
        ok = __all_sync(0xffffffffu, mbar_wait(c.own(), used & 1u, c.abort_flag)) && scores(0) && grads(0) &&
             __all_sync(0xffffffffu, mbar_wait(c.acc_empty(), (used & 1u) ^ 1u, c.abort_flag));
        ++used;
        for (int i = 0; i < n && ok; ++i) {
          ok = (i + 1 >= n || scores(i + 1)) && __all_sync(0xffffffffu, mbar_wait(c.ds(), (at + i) & 1u, c.abort_flag));
          if (!ok) break;
          tc_fence_after();
          ok = i + 1 >= n || grads(i + 1);
          if (!ok) break;
          if (one) {
            issue_ts<DP>(t_dq, tmem + ((at + i) & 1) * kTile, k_at(at + i), i > 0, a.head_dim);
            umma_commit(c.empty_a(at + i));
            if (i + 1 == n) { umma_commit(c.acc()); umma_commit(c.own_empty()); }
          }
        }
        at += n;
      }
      if (!ok && lane == 0) give_up(c, a.status);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ---------------- elements: one row per thread, half of the tile's keys per group ----------------
    const int half = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t dp_addr = t_dp + lanes + half * 64;
    bool ok = true;
    int at = 0, used = 0;
    while (ok && w.next()) {
      const KeyTiles<kTile> tiles = tiles_of();
      const int n = tiles.count(), rows = rows_of();
      const int pos = w.sq.shift + w.row0 + row;
      const bool mine = row < rows;
      const size_t place = (size_t)w.head * a.q_rows + w.sq.q0 + w.row0 + (mine ? row : 0);
      const float nl = mine ? -a.lse2[place] : -INFINITY, nd = mine ? -a.delta[place] : 0.f;
      const uint64_t neg_lse = pair2(nl, nl), neg_delta = pair2(nd, nd);
      const Score<CAP, BIAS> score(a, w.head);
      const RowKeys keys = row_keys(w.sq, a.causal, a.window, pos);
      for (int i = 0; i < n && ok; ++i, ++at) {
        const int j0 = tiles.at(i) * kTile + half * 64;
        // what the warp's rows see of these 64 keys: all, some (hidden ones become zeros), or nothing
        const int lo = keys.lo - j0, hi = keys.hi - j0, pre = keys.prefix - j0;
        const bool whole = __all_sync(0xffffffffu, (lo <= 0 && hi >= 64) || pre >= 64);
        const bool none = __all_sync(0xffffffffu, min(hi, 64) <= max(lo, 0) && pre <= 0);
        const uint32_t s_addr = tmem + (at & 1) * kTile + lanes + half * 64;
        ok = __all_sync(0xffffffffu, mbar_wait(c.s(at & 1), (at >> 1) & 1u, c.abort_flag));
        if (!ok) break;
        tc_fence_after();
        float pr[64];
        if (!none) {
          tmem_ld32(s_addr, *reinterpret_cast<uint32_t(*)[32]>(&pr[0]));
          tmem_ld32(s_addr + 32, *reinterpret_cast<uint32_t(*)[32]>(&pr[32]));
          tmem_ld_wait();
          const float d = (float)(pos - j0);
          score.cap(pr);
#pragma unroll
          for (int x = 0; x < 64; x += 2) {
            uint64_t cs;
            score.probs(pr[x], pr[x + 1], neg_lse, d - x, d - (x + 1), pr[x], pr[x + 1], cs);
            if (CAP) unpair2(mul2(pair2(pr[x], pr[x + 1]), cs), pr[x], pr[x + 1]);
          }
          if (!whole) {
#pragma unroll
            for (int b = 0; b < 64; b += 32) {
              const uint32_t seen = seen_bits(lo - b, hi - b, pre - b);
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if (!(seen & (1u << x))) pr[b + x] = 0.f;
            }
          }
        }
        ok = __all_sync(0xffffffffu, mbar_wait(c.dp(), at & 1u, c.abort_flag));
        if (!ok) break;
        tc_fence_after();
        if (none) {
          store_zeros(s_addr);
        } else {
#pragma unroll
          for (int c0 = 0; c0 < 2; ++c0) {
            float dp[32];
            tmem_ld32(dp_addr + c0 * 32, *reinterpret_cast<uint32_t(*)[32]>(&dp[0]));
            tmem_ld_wait();
            uint32_t pk[16];
#pragma unroll
            for (int x = 0; x < 32; x += 2) {
              float f0, f1;
              unpair2(mul2(add2(pair2(dp[x], dp[x + 1]), neg_delta), pair2(pr[c0 * 32 + x], pr[c0 * 32 + x + 1])), f0, f1);
              pk[x / 2] = bf16x2(f0, f1);
            }
            tmem_st16(s_addr + c0 * 16, pk);
          }
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(c.ds());
      }
      if (ok && n > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(c.acc(), used & 1u, c.abort_flag));
        ++used;
        tc_fence_after();
      }
      if (ok) {
        if (half == 0)
          store_row<DP>(t_dq + lanes, n > 0, c.acc_empty(), a.scale, mine,
                        reinterpret_cast<bf16*>(a.dq) + (size_t)(w.sq.q0 + w.row0 + (mine ? row : 0)) * a.q_stride +
                            (size_t)w.head * a.head_dim, a.head_dim);
      }
    }
    if (!ok && lane == 0) give_up(c, a.status);
  }
  block_end(c, tmem);
}

// delta = sum over the head of o * d_o, and the log-sum-exp in base 2 (+inf, i.e. p = 0, for rows that see nothing).
// Bound by reading o and d_o once: a block takes 8 rows of 32 heads, 16 lanes to a (row, head), with the loads of four
// of them in flight per lane; the results go through shared memory so that a head's 8 rows are written together.
constexpr int kDeltaRows = 8, kDeltaHeads = 32;
template <typename T>
__global__ void __launch_bounds__(256) attn_delta_kernel(AttnArgs a, float* lse2, float* delta) {
  constexpr int V = 16 / sizeof(T), ITEMS = 4, CHUNKS = sizeof(T) == 2 ? 1 : 2;   // a head is at most 128 values
  __shared__ float sums[kDeltaHeads * kDeltaRows];
  let_next_start();
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int head_blocks = (a.q_heads + kDeltaHeads - 1) / kDeltaHeads;
  const int row0 = blockIdx.x / head_blocks * kDeltaRows, head0 = blockIdx.x % head_blocks * kDeltaHeads;
#pragma unroll 1
  for (int i0 = 0; i0 < kDeltaRows * kDeltaHeads; i0 += 16 * ITEMS) {
    uint4 x[ITEMS][CHUNKS], y[ITEMS][CHUNKS];
#pragma unroll
    for (int n = 0; n < ITEMS; ++n) {
      const int i = i0 + n * 16 + g, row = row0 + i / kDeltaHeads, head = head0 + i % kDeltaHeads;
      const size_t at = (size_t)row * a.o_stride + (size_t)head * a.head_dim;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        const int c = (k * 16 + l) * V;
        const bool on = row < a.q_rows && head < a.q_heads && c < a.head_dim;
        x[n][k] = on ? *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.o) + at + c) : make_uint4(0, 0, 0, 0);
        y[n][k] = on ? *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.d_o) + at + c) : make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int n = 0; n < ITEMS; ++n) {
      const int i = i0 + n * 16 + g;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        const T* xe = reinterpret_cast<const T*>(&x[n][k]);
        const T* ye = reinterpret_cast<const T*>(&y[n][k]);
#pragma unroll
        for (int e = 0; e < V; ++e) sum += (float)xe[e] * (float)ye[e];
      }
#pragma unroll
      for (int f = 8; f >= 1; f >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, f);
      if (l == 0) sums[(i % kDeltaHeads) * kDeltaRows + i / kDeltaHeads] = sum;
    }
  }
  __syncthreads();
  const int head = head0 + threadIdx.x / kDeltaRows, row = row0 + threadIdx.x % kDeltaRows;
  if (head < a.q_heads && row < a.q_rows) {
    const size_t at = (size_t)head * a.q_rows + row;
    const float z = a.lse[at];
    delta[at] = sums[threadIdx.x];
    lse2[at] = z == -INFINITY ? INFINITY : z * kLog2e;
  }
  wait_for_last();                               // not needed here, but what comes behind this kernel needs the plan too
}

template <int DP, bool CAP, bool BIAS>
cudaError_t launch(const BwdParams& p, unsigned grid_kv, unsigned grid_q, cudaStream_t st) {
  static bool done_kv[64], done_q[64];
  cudaError_t e = allow_smem(attn_bwd_kv_kernel<DP, CAP, BIAS>, kSmemBytes<DP>, done_kv);
  if (e == cudaSuccess) e = allow_smem(attn_bwd_q_kernel<DP, CAP, BIAS>, kSmemBytes<DP>, done_q);
  if (e != cudaSuccess) return e;
  if (grid_kv) e = launch_behind(attn_bwd_kv_kernel<DP, CAP, BIAS>, grid_kv, kThreads, kSmemBytes<DP>, st, p);
  if (e == cudaSuccess && grid_q)
    e = launch_behind(attn_bwd_q_kernel<DP, CAP, BIAS>, grid_q, kThreads, kSmemBytes<DP>, st, p);
  return e;
}
template <int DP>
cudaError_t launch_dp(const BwdParams& p, unsigned gk, unsigned gq, cudaStream_t st) {
  if (p.a.softcap > 0.f) return p.a.slopes ? launch<DP, true, true>(p, gk, gq, st) : launch<DP, true, false>(p, gk, gq, st);
  return p.a.slopes ? launch<DP, false, true>(p, gk, gq, st) : launch<DP, false, false>(p, gk, gq, st);
}

}  // namespace

cudaError_t launch_attn_delta(const AttnArgs& a, bool bf16_mode, float* lse2, float* delta, cudaStream_t st) {
  const long long blocks = ((long long)a.q_rows + kDeltaRows - 1) / kDeltaRows * ((a.q_heads + kDeltaHeads - 1) / kDeltaHeads);
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  if (blocks == 0) return cudaSuccess;
  if (bf16_mode) return launch_behind(attn_delta_kernel<bf16>, (unsigned)blocks, 256, 0, st, a, lse2, delta);
  attn_delta_kernel<float><<<(unsigned)blocks, 256, 0, st>>>(a, lse2, delta);
  return cudaGetLastError();
}

cudaError_t launch_attn_backward_tc(const AttnArgs& a, cudaStream_t st) {
  BwdParams p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  const long long qr = a.q_rows > 0 ? a.q_rows : 1, kr = a.k_rows > 0 ? a.k_rows : 1;   // without rows no tile is loaded
  if (!tc_encode_heads(&p.q_map, a.q, qr, a.q_heads, a.head_dim, a.q_stride, kTile) ||
      !tc_encode_heads(&p.do_map, a.d_o, qr, a.q_heads, a.head_dim, a.o_stride, kTile) ||
      !tc_encode_heads(&p.k_map, a.k, kr, a.kv_heads, a.head_dim, a.k_stride, kTile) ||
      !tc_encode_heads(&p.v_map, a.v, kr, a.kv_heads, a.head_dim, a.v_stride, kTile))
    return cudaErrorInvalidValue;
  long long gk = a.k_rows ? ((long long)(a.k_rows + kBwdTile - 1) / kBwdTile + a.n_seqs) * a.kv_heads : 0;
  long long gq = a.q_rows ? ((long long)(a.q_rows + kBwdTile - 1) / kBwdTile + a.n_seqs) * a.q_heads : 0;
  if (gk > 0x7fff0000LL || gq > 0x7fff0000LL) return cudaErrorInvalidValue;
  const int sms = attn_sm_count();                           // one block per SM, which walks over the tiles
  if (gk > sms) gk = sms;
  if (gq > sms) gq = sms;
  return a.head_dim <= 64 ? launch_dp<64>(p, (unsigned)gk, (unsigned)gq, st) : launch_dp<128>(p, (unsigned)gk, (unsigned)gq, st);
}

}  // namespace mixlora
