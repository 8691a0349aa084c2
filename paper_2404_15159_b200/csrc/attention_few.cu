// Masked attention for few query rows of each sequence (a decoding step): bound by reading the keys and values once.
//
// The rows of a sequence that share a key head (its query heads times the sequence's new tokens) are the 16 rows of one
// m16n8k16 product, so that every key and value is read once for all of them (more rows go to several blocks, which find
// the keys in L2).  mma.sync and not tcgen05: a tile of 128 rows would hold 1 to 16, and the product takes a few per cent
// of the time that the keys take to arrive.  The keys of a (sequence, key head) are split over several blocks where there
// are few of those, which join their (m, l, sum p v) in index order.
// Measured: 64 sequences in slots of 8192 keys, 32 / 8 heads of 128, 1.21 GB: 184 us (6.6 TB/s) and 5 us for the join; one
// sequence of 1000 keys, 32 heads: 8 us; fp32, 7 sequences of 4 tokens and up to 2000 keys, 16 / 8 heads of 64: 18 us, where
// no load is under way while a step is computed.
#include "attention.cuh"

namespace mixlora {
namespace {

constexpr int kWarps = 4;
constexpr int kStep = 16;                        // keys per step of a warp
constexpr int kStages = 3;

constexpr int kClusterMax = 8;                   // a cluster's blocks, in every configuration

struct FewParams {
  AttnArgs a;
  float* part;                                   // [seq, key head, chunk, split, 16 rows, head_dim + 3]: sum p v, m (base
                                                 // 2), sum p as taken and as rounded
  int splits, rows, chunks;                      // rows = group * max_q_len, in chunks of kFewRows
  bool cluster;                                  // the splits of a (sequence, key head) are one cluster
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes to shared memory; zeros where `on` is false (nothing is read then)
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The block's (sequence, key head, split), and the key groups of kStep keys it works on.
struct Share {
  AttnSeq sq;
  int seq, kvh, split, lq;
  int row0, rows;                                // the block's chunk of the rows
  KeyTiles<kStep> tiles;
  int t0, t1;
};
__device__ __forceinline__ Share block_share(const FewParams& p) {
  const AttnArgs& a = p.a;
  Share w;
  w.split = blockIdx.x % p.splits;
  int rest = blockIdx.x / p.splits;
  w.row0 = rest % p.chunks * kFewRows;
  w.rows = min(kFewRows, p.rows - w.row0);
  rest /= p.chunks;
  w.kvh = rest % a.kv_heads;
  w.seq = rest / a.kv_heads;
  w.sq = load_seq(a, w.seq);
  w.lq = min(w.sq.lq, a.max_q_len);
  w.t0 = w.t1 = 0;
  w.tiles = KeyTiles<kStep>{0, 0, 0};
  if (w.lq > 0) {
    w.tiles = key_tiles<kStep>(w.sq, a.causal, a.window, w.sq.shift, w.sq.shift + w.lq - 1);
    const long long n = w.tiles.count();
    w.t0 = (int)(n * w.split / p.splits);
    w.t1 = (int)(n * (w.split + 1) / p.splits);
  }
  return w;
}

template <bool CAP, bool BIAS>
struct ScoreMap {
  float mul, cap2;
  __device__ __forceinline__ explicit ScoreMap(const AttnArgs& a)
      : mul(CAP ? a.scale / a.softcap : a.scale * kLog2e), cap2(a.softcap * kLog2e) {}
  // score in base 2; `slope2` in base 2 too
  __device__ __forceinline__ float operator()(float s, float slope2, int distance) const {
    float x = s * mul;
    if (CAP) x = cap2 * tanh_one(x);
    if (BIAS) x -= slope2 * fabsf((float)distance);
    return x;
  }
};

// A row's result: o over the sum of the p it was made with, and the log-sum-exp
template <typename T>
__device__ __forceinline__ void write_result(const FewParams& p, const Share& w, int qi, int head, int c, float o, float l,
                                             float u, float m) {
  const AttnArgs& a = p.a;
  const size_t row = (size_t)(w.sq.q0 + qi);
  const float inv = l > 0.f || l != l ? 1.f / u : 0.f;
  T* out = reinterpret_cast<T*>(a.out) + row * a.o_stride + (size_t)head * a.head_dim + c;
  if constexpr (sizeof(T) == 2) *out = __float2bfloat16(o * inv);
  else *out = o * inv;
  if (c == 0 && a.lse) a.lse[(size_t)head * a.q_rows + row] = (m + log2f(l)) * kLn2;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A value at this shared-memory address in block `rank` of the cluster
__device__ __forceinline__ float load_from(const float* mine, int rank) {
  uint32_t addr;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_addr(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// Joins the states of a block's warps in order, then the splits in index order: through the cluster's shared memory,
// or through a partial in the workspace and a second launch.
// `st_m`, `st_l`, `st_u` [states][16], `st_o` [states][16][DP] in shared memory; the block's own sums go over the first state's.
template <typename T>
__device__ __forceinline__ void finish_block(const FewParams& p, const Share& w, float* st_m, float* st_l, float* st_u,
                                             float* st_o, int dp, int states) {
  const AttnArgs& a = p.a;
  const int d = a.head_dim;
  const bool cluster = p.cluster;
  // a thread owns the same (row, value)s in all passes, but reads every warp's m and l of its rows
  float keep_m = -INFINITY, keep_l = 0.f, keep_u = 0.f;
  if (threadIdx.x < 16) {
    float m = -INFINITY, l = 0.f, u = 0.f;
    for (int x = 0; x < states; ++x) m = fmaxf(m, st_m[x * 16 + threadIdx.x]);
    for (int x = 0; x < states; ++x) {
      const float mx = st_m[x * 16 + threadIdx.x], f = mx == -INFINITY ? 0.f : ex2(mx - m);
      l += f * st_l[x * 16 + threadIdx.x];
      u += f * st_u[x * 16 + threadIdx.x];
    }
    keep_m = m;
    keep_l = l;
    keep_u = u;
  }
  for (int i = threadIdx.x; i < w.rows * d; i += kWarps * 32) {
    const int r = i / d, c = i - r * d;
    float m = -INFINITY, o = 0.f;
    for (int x = 0; x < states; ++x) m = fmaxf(m, st_m[x * 16 + r]);
    for (int x = 0; x < states; ++x) {
      const float f = st_m[x * 16 + r] == -INFINITY ? 0.f : ex2(st_m[x * 16 + r] - m);
      o += f * st_o[(x * 16 + r) * dp + c];
    }
    st_o[r * dp + c] = o;
  }
  __syncthreads();
  if (threadIdx.x < 16) { st_m[threadIdx.x] = keep_m; st_l[threadIdx.x] = keep_l; st_u[threadIdx.x] = keep_u; }
  if (cluster) cluster_sync();
  else __syncthreads();
  // the cluster's blocks share the row's values out among themselves
  const int first = cluster ? w.split : 0, step = cluster ? p.splits : 1;
  for (int i = threadIdx.x + first * kWarps * 32; i < w.rows * d; i += step * kWarps * 32) {
    const int r = i / d, c = i - r * d;
    const int qi = (w.row0 + r) / a.group, head = w.kvh * a.group + (w.row0 + r - qi * a.group);
    if (qi >= w.lq) continue;
    float m = st_m[r], l = st_l[r], u = st_u[r], o = st_o[r * dp + c];
    if (cluster) {
      float ms[kClusterMax];
      m = -INFINITY;
#pragma unroll
      for (int s = 0; s < kClusterMax; ++s) {
        ms[s] = s < p.splits ? load_from(st_m + r, s) : -INFINITY;
        m = fmaxf(m, ms[s]);
      }
      l = u = o = 0.f;
#pragma unroll
      for (int s = 0; s < kClusterMax; ++s)
        if (s < p.splits && ms[s] != -INFINITY) {
          const float f = ex2(ms[s] - m);
          l += f * load_from(st_l + r, s);
          u += f * load_from(st_u + r, s);
          o += f * load_from(st_o + r * dp + c, s);
        }
    }
    if (p.splits > 1 && !cluster) {
      const size_t block = (((size_t)w.seq * a.kv_heads + w.kvh) * p.chunks + w.row0 / kFewRows) * p.splits + w.split;
      float* dst = p.part + (block * kFewRows + r) * (d + 3);
      dst[c] = o;
      if (c == 0) { dst[d] = m; dst[d + 1] = l; dst[d + 2] = u; }
    } else {
      write_result<T>(p, w, qi, head, c, o, l, u, m);
    }
  }
  if (cluster) cluster_sync();                   // nobody leaves while its shared memory is read
}

// bf16.  A warp takes every kWarps-th group of 16 keys; K and V of the next groups travel through its own ring of
// kStages stages in shared memory (16-byte pieces, XORed with the key so that the 8 rows of an ldmatrix fall into
// different banks).  Keys behind the last one are never read: their rows are filled with zeros.
//
// p goes into its product in bf16, and o is divided by the sum of the rounded p.  With at most 8 rows (TWO) rows 8 to 15 of
// the product are empty and take what the rounding left of rows 0 to 7, again in bf16: p then keeps 16 bits, and both halves
// of the result are added up at the end (64 sequences of up to 8192 keys, 4 rows: the same 213 us as with p rounded once,
// the error against 64 bits 0.0024 -> 0.0017, which is the output's own rounding).  More rows would need a second product
// (16 rows 231 -> 249 us, 32 rows 351 -> 418), so there a weight is rounded once, by half a step, 2^-8 of itself.
template <int DP, bool CAP, bool BIAS, bool TWO>
__global__ void __launch_bounds__(kWarps * 32, 2) attn_few_bf16_kernel(FewParams p) {
  constexpr int C = DP / 8;                      // 16-byte pieces of a row
  constexpr int kStageBytes = 2 * kStep * DP * 2;
  extern __shared__ __align__(128) uint8_t smem[];
  const AttnArgs& a = p.a;
  let_next_start();
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) *a.status = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const Share w = block_share(p);
  const int d = a.head_dim;
  const uint32_t ring = smem_addr(smem) + warp * kStages * kStageBytes;
  const bf16* kp = reinterpret_cast<const bf16*>(a.k) + (size_t)w.kvh * d;
  const bf16* vp = reinterpret_cast<const bf16*>(a.v) + (size_t)w.kvh * d;

  const int first = w.t0 + warp, n = first < w.t1 ? (w.t1 - first + kWarps - 1) / kWarps : 0;
  auto load = [&](int i) {
    if (i < n) {
      const int j0 = w.tiles.at(first + i * kWarps) * kStep;
      const uint32_t dst = ring + (i % kStages) * kStageBytes;
#pragma unroll
      for (int x = 0; x < kStep * C / 32; ++x) {
        const int idx = x * 32 + lane, r = idx / C, c = idx % C;
        const bool on = j0 + r < w.sq.lk && c * 8 < d;
        const size_t row = (size_t)(w.sq.k0 + (on ? j0 + r : 0));
        const int at = on ? c * 8 : 0;
        const uint32_t off = (uint32_t)(r * DP * 2 + ((c ^ (r & 7)) << 4));
        copy16(dst + off, kp + row * a.k_stride + at, on);
        copy16(dst + kStep * DP * 2 + off, vp + row * a.v_stride + at, on);
      }
    }
    copy_commit();
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) load(i);

  // the queries' fragments, straight from memory: rows r = qi * group + head, zeros behind the last
  uint32_t qf[DP / 16][4];
  RowKeys keys[2];
  float slope2[2] = {0.f, 0.f};
  int pos[2];
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    const int r = w.row0 + g + 8 * hf, qi = r / a.group, hd = w.kvh * a.group + (r - qi * a.group);
    const bool on = g + 8 * hf < w.rows && qi < w.lq;
    pos[hf] = w.sq.shift + qi;
    keys[hf] = on ? row_keys(w.sq, a.causal, a.window, pos[hf]) : RowKeys{0, 0, 0};
    if (BIAS && on) slope2[hf] = a.slopes[hd] * kLog2e;
    const bf16* src = reinterpret_cast<const bf16*>(a.q) + (size_t)(w.sq.q0 + (on ? qi : 0)) * a.q_stride + (size_t)hd * d;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int c = k * 16 + u * 8 + 2 * t;
        qf[k][hf + 2 * u] = on && c < d ? *reinterpret_cast<const uint32_t*>(src + c) : 0u;
      }
  }

  const ScoreMap<CAP, BIAS> score(a);
  float o[DP / 8][4];
#pragma unroll
  for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, used[2] = {0.f, 0.f};   // sums of p as taken and as rounded
  for (int i = 0; i < n; ++i) {
    load(i + kStages - 1);
    copy_wait<kStages - 1>();
    __syncwarp();
    const uint32_t kb = ring + (i % kStages) * kStageBytes, vb = kb + kStep * DP * 2;
    float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    {
      // matrices of an ldmatrix: keys 0-7 | 0-7 | 8-15 | 8-15, values 0-7 | 8-15 | 0-7 | 8-15 of the step
      const int r = (lane & 7) + ((lane >> 4) << 3), hi = (lane >> 3) & 1;
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) {
        uint32_t b[4];
        ldsm4(kb + r * DP * 2 + (((2 * k + hi) ^ (r & 7)) << 4), b);
        mma16816(s[0], qf[k], b[0], b[1]);
        mma16816(s[1], qf[k], b[2], b[3]);
      }
    }
    const int j0 = w.tiles.at(first + i * kWarps) * kStep;
    float mt[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      if (hf && TWO) break;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int j = j0 + (x >> 1) * 8 + 2 * t + (x & 1);
        float& v = s[x >> 1][2 * hf + (x & 1)];
        v = score(v, slope2[hf], pos[hf] - j);
        if (!keys[hf].sees(j)) v = -INFINITY;
        mt[hf] = fmaxf(mt[hf], v);
      }
      mt[hf] = fmaxf(mt[hf], __shfl_xor_sync(0xffffffffu, mt[hf], 1));
      mt[hf] = fmaxf(mt[hf], __shfl_xor_sync(0xffffffffu, mt[hf], 2));
    }
    // as in the tiled kernel, a row's maximum moves only where it has grown by more than 2^8
    const bool grown = (mt[0] > m[0] && mt[0] - m[0] > 8.f) || (mt[1] > m[1] && mt[1] - m[1] > 8.f);
    if (__any_sync(0xffffffffu, grown)) {
      float f[2];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const float mn = fmaxf(m[hf], mt[hf]);
        f[hf] = m[hf] == -INFINITY ? 0.f : ex2(m[hf] - mn);
        m[hf] = mn;
        l[hf] *= f[hf];
        used[hf] *= f[hf];
        if (hf && TWO) f[1] = f[0];
#pragma unroll
        for (int x = 0; x < DP / 8; ++x) { o[x][2 * hf] *= f[hf]; o[x][2 * hf + 1] *= f[hf]; }
      }
    }
    uint32_t pf[4];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      if (hf && TWO) break;
      const float base = m[hf] == -INFINITY ? 0.f : m[hf];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float e0 = ex2(s[u][2 * hf] - base), e1 = ex2(s[u][2 * hf + 1] - base);
        l[hf] += e0 + e1;
        const uint32_t r = bf16x2(e0, e1);
        pf[hf + 2 * u] = r;
        if (TWO) pf[1 + 2 * u] = bf16x2(e0 - bf16_lo(r), e1 - bf16_hi(r));
        else used[hf] += bf16_lo(r) + bf16_hi(r);
      }
    }
    {
      // matrices: keys 0-7 | 8-15 | 0-7 | 8-15, values of two neighbouring 8-value pieces
      const int r = lane & 15, hi = lane >> 4;
#pragma unroll
      for (int x = 0; x < DP / 16; ++x) {
        uint32_t b[4];
        ldsm4t(vb + r * DP * 2 + (((2 * x + hi) ^ (r & 7)) << 4), b);
        mma16816(o[2 * x], pf, b[0], b[1]);
        mma16816(o[2 * x + 1], pf, b[2], b[3]);
      }
    }
    __syncwarp();                                // the stage may be filled again
  }
  copy_wait<0>();
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    l[hf] += __shfl_xor_sync(0xffffffffu, l[hf], 1);
    l[hf] += __shfl_xor_sync(0xffffffffu, l[hf], 2);
    used[hf] += __shfl_xor_sync(0xffffffffu, used[hf], 1);
    used[hf] += __shfl_xor_sync(0xffffffffu, used[hf], 2);
  }
  if (TWO) {
    used[0] = l[0];
#pragma unroll
    for (int x = 0; x < DP / 8; ++x) { o[x][0] += o[x][2]; o[x][1] += o[x][3]; }
  }
  __syncthreads();                               // the rings become the block's exchange
  float* st_m = reinterpret_cast<float*>(smem);
  float* st_l = st_m + kWarps * 16;
  float* st_u = st_l + kWarps * 16;
  float* st_o = st_u + kWarps * 16;
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    const int r = g + 8 * hf;
    if (t == 0) { st_m[warp * 16 + r] = m[hf]; st_l[warp * 16 + r] = l[hf]; st_u[warp * 16 + r] = used[hf]; }
#pragma unroll
    for (int x = 0; x < DP / 8; ++x)
      *reinterpret_cast<float2*>(st_o + (warp * 16 + r) * DP + x * 8 + 2 * t) = make_float2(o[x][2 * hf], o[x][2 * hf + 1]);
  }
  __syncthreads();
  finish_block<bf16>(p, w, st_m, st_l, st_u, st_o, DP, kWarps);
}

// Where a value of a batch ends up when the M partial sums of LPK lanes are added up: every step of the exchange halves the
// values a lane keeps (the upper half in lanes with that bit set) until one is left, later steps only add.
template <int LPK, int M>
struct Spread {
  static constexpr int kOwn = M > LPK ? M / LPK : 1;         // values of a lane in the end
  // the lane (of LPK) that ends up with value `idx`, and which of its values it is
  static __host__ __device__ constexpr int lane_of(int idx) {
    int lane = 0, cur = M;
    for (int off = LPK / 2; off >= 1; off >>= 1)
      if (cur > 1) {
        cur >>= 1;
        if (idx & cur) lane |= off;
      }
    return lane;
  }
  static __device__ __forceinline__ int first_of(int lane) {
    int idx = 0, cur = M;
#pragma unroll
    for (int off = LPK / 2; off >= 1; off >>= 1)
      if (cur > 1) {
        cur >>= 1;
        if (lane & off) idx |= cur;
      }
    return idx;
  }
  static __device__ __forceinline__ void add_up(float (&v)[M], int lane) {
    int cur = M;
#pragma unroll
    for (int off = LPK / 2; off >= 1; off >>= 1) {
      if (cur > 1) {
        cur >>= 1;
        const bool up = lane & off;
#pragma unroll
        for (int k = 0; k < M / 2; ++k)
          if (k < cur) {
            const float send = up ? v[k] : v[k + cur], keep = up ? v[k + cur] : v[k];
            v[k] = keep + __shfl_xor_sync(0xffffffffu, send, off);
          }
      } else {
        v[0] += __shfl_xor_sync(0xffffffffu, v[0], off);
      }
    }
  }
  // over the lanes that hold the four keys of a row (values 4 r .. 4 r + 3)
  template <typename F>
  static __device__ __forceinline__ float over_keys(float v, F f) {
    int cur = M;
#pragma unroll
    for (int off = LPK / 2; off >= 1; off >>= 1)
      if (cur > 1) {
        cur >>= 1;
        if (cur < 4) v = f(v, __shfl_xor_sync(0xffffffffu, v, off));
      }
    return v;
  }
};

// fp32.  LPK lanes hold a key (4 values each), and four keys at a time; their ROWS x 4 scores are summed so that every
// lane ends up with its own share of them, whose exponentials it takes once and hands back to the others.  The cap goes
// through tanhf: this is the check mode.
template <int LPK, int ROWS, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kWarps * 32) attn_few_f32_kernel(FewParams p) {
  constexpr int SUB = 32 / LPK, DP = LPK * 4, M = 4 * ROWS;
  using S = Spread<LPK, M>;
  constexpr int OWN = S::kOwn;
  extern __shared__ __align__(128) uint8_t smem[];
  const AttnArgs& a = p.a;
  let_next_start();
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) *a.status = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = lane / LPK, sl = lane % LPK, c = sl * 4;
  const Share w = block_share(p);
  const int d = a.head_dim;
  const bool on_c = c < d;
  const float* kp = reinterpret_cast<const float*>(a.k) + (size_t)w.kvh * d + (on_c ? c : 0);
  const float* vp = reinterpret_cast<const float*>(a.v) + (size_t)w.kvh * d + (on_c ? c : 0);
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);

  float4 q[ROWS], o[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int qi = (w.row0 + r) / a.group, hd = w.kvh * a.group + (w.row0 + r - qi * a.group);
    const bool on = r < w.rows && qi < w.lq;
    q[r] = on && on_c ? *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) +
                                                          (size_t)(w.sq.q0 + qi) * a.q_stride + (size_t)hd * d + c)
                      : zero;
    o[r] = zero;
  }
  // this lane's row, the first of its keys, and the row's running maximum and part of the sum
  const int own = S::first_of(sl), own_r = own >> 2, own_x = own & 3;
  const int qi = (w.row0 + own_r) / a.group, hd = w.kvh * a.group + (w.row0 + own_r - qi * a.group);
  const bool live = own_r < w.rows && qi < w.lq;
  const int pos = w.sq.shift + qi;
  const RowKeys keys = live ? row_keys(w.sq, a.causal, a.window, pos) : RowKeys{0, 0, 0};
  const float slope2 = BIAS && live ? a.slopes[hd] * kLog2e : 0.f;
  float m = -INFINITY, l = 0.f;
  auto larger = [](float x, float y) { return fmaxf(x, y); };
  auto sum = [](float x, float y) { return x + y; };

  for (int tt = w.t0 + warp; tt < w.t1; tt += kWarps) {
    const int j0 = w.tiles.at(tt) * kStep;
#pragma unroll
    for (int b = 0; b < kStep / (4 * SUB); ++b) {
      const int jb = j0 + (b * SUB + sub) * 4;   // this group of lanes' four keys
      float4 k[4], v[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool on = on_c && jb + x < w.sq.lk;
        const size_t row = (size_t)(w.sq.k0 + (on ? jb + x : 0));
        k[x] = on ? *reinterpret_cast<const float4*>(kp + row * a.k_stride) : zero;
        v[x] = on ? *reinterpret_cast<const float4*>(vp + row * a.v_stride) : zero;
      }
      float s[M];
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          s[4 * r + x] = fmaf(q[r].w, k[x].w, fmaf(q[r].z, k[x].z, fmaf(q[r].y, k[x].y, q[r].x * k[x].x)));
      S::add_up(s, sl);
      float mt = -INFINITY;
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        const int j = jb + own_x + i;
        float y = s[i] * a.scale;
        if (CAP) y = a.softcap * tanhf(y / a.softcap);
        y *= kLog2e;
        if (BIAS) y -= slope2 * fabsf((float)(pos - j));
        s[i] = keys.sees(j) ? y : -INFINITY;
        mt = fmaxf(mt, s[i]);
      }
      mt = S::over_keys(mt, larger);
      const bool grown = mt > m + 8.f || (mt > m && m == -INFINITY);
      if (__any_sync(0xffffffffu, grown)) {
        const float m_new = grown ? mt : m, f = m == -INFINITY ? 0.f : exp2f(m - m_new);
        m = m_new;
        l *= f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          const float fr = __shfl_sync(0xffffffffu, f, sub * LPK + S::lane_of(4 * r));
          o[r].x *= fr; o[r].y *= fr; o[r].z *= fr; o[r].w *= fr;
        }
      }
      const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        s[i] = exp2f(s[i] - base);
        l += s[i];
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float e = __shfl_sync(0xffffffffu, s[(4 * r + x) % OWN], sub * LPK + S::lane_of(4 * r + x));
          o[r].x = fmaf(e, v[x].x, o[r].x);
          o[r].y = fmaf(e, v[x].y, o[r].y);
          o[r].z = fmaf(e, v[x].z, o[r].z);
          o[r].w = fmaf(e, v[x].w, o[r].w);
        }
    }
  }
  constexpr int kStates = kWarps * SUB;
  float* st_m = reinterpret_cast<float*>(smem);
  float* st_l = st_m + kStates * 16;
  float* st_u = st_l + kStates * 16;              // p is used as taken
  float* st_o = st_u + kStates * 16;
  const int state = warp * SUB + sub;
  l = S::over_keys(l, sum);
  if (own_x == 0) st_m[state * 16 + own_r] = m, st_l[state * 16 + own_r] = l, st_u[state * 16 + own_r] = l;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) *reinterpret_cast<float4*>(st_o + (state * 16 + r) * DP + c) = o[r];
  __syncthreads();
  finish_block<float>(p, w, st_m, st_l, st_u, st_o, DP, kStates);
}

// Joins the splits of a row in index order; one warp per (sequence, query, head).
template <typename T>
__global__ void __launch_bounds__(128) attn_few_join_kernel(FewParams p) {
  const AttnArgs& a = p.a;
  wait_for_last();
  const int item = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int seq = item / (p.rows * a.kv_heads);
  if (seq >= a.n_seqs) return;
  const int rest = item - seq * p.rows * a.kv_heads, kvh = rest / p.rows, r = rest - kvh * p.rows;
  const int qi = r / a.group, head = kvh * a.group + (r - qi * a.group), d = a.head_dim;
  const int q0 = clamp_int(a.q_off[seq], 0, a.q_rows);
  if (qi >= min(seq_rows(a.q_off, seq, a.q_rows), a.max_q_len)) return;
  const size_t pitch = (size_t)kFewRows * (d + 3);
  const float* src = p.part + (((size_t)seq * a.kv_heads + kvh) * p.chunks + r / kFewRows) * p.splits * pitch +
                     (size_t)(r % kFewRows) * (d + 3);
  float m = -INFINITY;
  for (int s = lane; s < p.splits; s += 32) m = fmaxf(m, src[s * pitch + d]);
#pragma unroll
  for (int f = 16; f >= 1; f >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, f));
  float l = 0.f, u = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < p.splits; ++s) {
    const float ms = src[s * pitch + d];
    const float f = ms == -INFINITY ? 0.f : exp2f(ms - m);
    l += f * src[s * pitch + d + 1];
    u += f * src[s * pitch + d + 2];
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (lane + 32 * x < d) o[x] += f * src[s * pitch + lane + 32 * x];
  }
  const float inv = l > 0.f || l != l ? 1.f / u : 0.f;
  T* out = reinterpret_cast<T*>(a.out) + (size_t)(q0 + qi) * a.o_stride + (size_t)head * d;
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (lane + 32 * x < d) {
      if constexpr (sizeof(T) == 2) out[lane + 32 * x] = __float2bfloat16(o[x] * inv);
      else out[lane + 32 * x] = o[x] * inv;
    }
  if (lane == 0 && a.lse) a.lse[(size_t)head * a.q_rows + q0 + qi] = (m + log2f(l)) * kLn2;
}

constexpr size_t exchange_bytes(int dp, int states) { return (size_t)states * 16 * (dp + 3) * 4; }

template <typename K>
cudaError_t launch_blocks(K kernel, const FewParams& p, unsigned grid, size_t smem, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.splits;             // a (sequence, key head)'s splits are neighbouring blocks
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.cluster ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <int DP, bool CAP, bool BIAS, bool TWO>
cudaError_t launch_bf16(const FewParams& p, unsigned grid, cudaStream_t st) {
  constexpr size_t ring = (size_t)kWarps * kStages * 2 * kStep * DP * 2;
  constexpr size_t smem = ring > exchange_bytes(DP, kWarps) ? ring : exchange_bytes(DP, kWarps);
  static bool done[64];
  cudaError_t e = allow_smem(attn_few_bf16_kernel<DP, CAP, BIAS, TWO>, (int)smem, done);
  if (e != cudaSuccess) return e;
  return launch_blocks(attn_few_bf16_kernel<DP, CAP, BIAS, TWO>, p, grid, smem, st);
}
template <int LPK, int ROWS, bool CAP, bool BIAS>
cudaError_t launch_f32(const FewParams& p, unsigned grid, cudaStream_t st) {
  return launch_blocks(attn_few_f32_kernel<LPK, ROWS, CAP, BIAS>, p, grid, exchange_bytes(LPK * 4, kWarps * (32 / LPK)), st);
}
template <bool CAP, bool BIAS>
cudaError_t launch_mode(const FewParams& p, bool bf16_mode, unsigned grid, cudaStream_t st) {
  const bool narrow = p.a.head_dim <= 64;
  if (bf16_mode && p.rows <= 8)
    return narrow ? launch_bf16<64, CAP, BIAS, true>(p, grid, st) : launch_bf16<128, CAP, BIAS, true>(p, grid, st);
  if (bf16_mode) return narrow ? launch_bf16<64, CAP, BIAS, false>(p, grid, st) : launch_bf16<128, CAP, BIAS, false>(p, grid, st);
  // the rows are registers: as few as hold them
  if (p.rows <= 1) return narrow ? launch_f32<16, 1, CAP, BIAS>(p, grid, st) : launch_f32<32, 1, CAP, BIAS>(p, grid, st);
  if (p.rows <= 4) return narrow ? launch_f32<16, 4, CAP, BIAS>(p, grid, st) : launch_f32<32, 4, CAP, BIAS>(p, grid, st);
  if (p.rows <= 8) return narrow ? launch_f32<16, 8, CAP, BIAS>(p, grid, st) : launch_f32<32, 8, CAP, BIAS>(p, grid, st);
  return narrow ? launch_f32<16, 16, CAP, BIAS>(p, grid, st) : launch_f32<32, 16, CAP, BIAS>(p, grid, st);
}

}  // namespace

// Splits of a (sequence, key head), none under 256 keys.  Where the 2 x 148 blocks that run together are not reached
// without splitting, and are with at most 8, the splits are one cluster and join in the same launch (a call on one
// sequence of 1024 keys, 32 heads: 8 us, and 10 with a second launch).  Else there are enough for about four rounds of
// blocks (lengths differ, and short pieces even that out), joined by a second launch (64 sequences of up to 8192 keys:
// 186 us; clusters, which wait for a free group of SMs, 190).
FewSplits attn_few_splits(int n_seqs, int kv_heads, int rows, long long k_rows, int max_k_len) {
  const long long pairs = (long long)n_seqs * kv_heads * ((rows + kFewRows - 1) / kFewRows);
  if (pairs <= 0) return FewSplits{1, false};
  long long longest = max_k_len > 0 ? max_k_len : (k_rows + n_seqs - 1) / n_seqs;
  if (longest > k_rows) longest = k_rows;
  const long long cap = longest > 256 ? (longest + 255) / 256 : 1;
  auto fill = [&](long long blocks) {
    const long long s = (blocks + pairs - 1) / pairs;
    return s < cap ? s : cap;
  };
  const long long few = fill(2 * 148);
  if (few <= 1 && pairs < 2 * 148) return FewSplits{1, false};
  if (few > 1 && few <= kClusterMax) return FewSplits{(int)few, true};
  const long long many = fill(4 * 2 * 148);
  return FewSplits{(int)(many < 256 ? many : 256), false};
}

cudaError_t launch_attn_few(const AttnArgs& a, bool bf16_mode, FewSplits splits, float* part, cudaStream_t st) {
  const int rows = a.group * a.max_q_len;
  FewParams p{a, part, splits.count, rows, (rows + kFewRows - 1) / kFewRows, splits.cluster};
  const long long blocks = (long long)a.n_seqs * a.kv_heads * p.chunks * p.splits;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  const unsigned grid = (unsigned)blocks;
  cudaError_t e;
  if (a.softcap > 0.f) e = a.slopes ? launch_mode<true, true>(p, bf16_mode, grid, st) : launch_mode<true, false>(p, bf16_mode, grid, st);
  else e = a.slopes ? launch_mode<false, true>(p, bf16_mode, grid, st) : launch_mode<false, false>(p, bf16_mode, grid, st);
  if (e != cudaSuccess || p.splits == 1 || p.cluster) return e;
  const long long items = (long long)a.n_seqs * a.kv_heads * p.rows;
  const unsigned jg = (unsigned)((items + 3) / 4);
  return bf16_mode ? launch_behind(attn_few_join_kernel<bf16>, jg, 128, 0, st, p)
                   : launch_behind(attn_few_join_kernel<float>, jg, 128, 0, st, p);
}

}  // namespace mixlora
