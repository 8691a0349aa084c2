// Shared parts of the attention kernels: arguments, the sequences' geometry, which keys a query sees.
#pragma once

#include "common.cuh"

namespace mixlora {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// One sequence: its rows and keys, and the position of its first row (query row i has position shift + i; key j has
// position j, so that the last row stands at the last key).  Offsets come from device memory and are held inside the
// tensors whatever they say.
struct AttnSeq {
  int q0, lq, k0, lk, shift, prefix;
};
// A tile of query rows or keys: its sequence and its first row (key) in it.
struct alignas(32) AttnTile {
  AttnSeq sq;
  int row0, pad;
};

struct AttnArgs {
  const void *q, *k, *v;          // [rows, heads, head_dim], `*_stride` elements from row to row
  const void *o, *d_o;            // backward: the forward's output and its gradient, both with o's stride
  void* out;                      // forward: o
  void *dq, *dk, *dv;             // strides of q, k, v
  float* lse;                     // [q_heads, q_rows], natural logarithm
  const float* lse2;              // backward: lse in base 2, +inf for rows that see nothing   [q_heads, q_rows]
  const float* delta;             // backward: sum over head_dim of o * d_o                    [q_heads, q_rows]
  const int32_t *q_off, *k_off;   // [n_seqs + 1]
  const int32_t *k_len, *prefix;  // [n_seqs] or NULL
  const AttnTile *q_tiles, *k_tiles;  // tensor-core kernels: the planned tiles, longest work first, and their numbers
  const int32_t *n_q_tiles, *n_k_tiles;
  const float* slopes;            // [q_heads] or NULL
  int32_t* status;
  long long q_stride, k_stride, v_stride, o_stride;
  int n_seqs, q_rows, k_rows, q_heads, kv_heads, group, head_dim;
  int causal, window, max_q_len;
  float scale;                    // multiplies q . k
  float softcap;                  // > 0: scores become softcap * tanh(score / softcap)
};

__device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return min(max(v, lo), hi); }

__device__ __forceinline__ int seq_rows(const int32_t* off, int b, int rows) {
  const int a = clamp_int(off[b], 0, rows);
  return clamp_int(off[b + 1], a, rows) - a;
}

__device__ __forceinline__ AttnSeq load_seq(const AttnArgs& p, int b) {
  AttnSeq s;
  s.q0 = clamp_int(p.q_off[b], 0, p.q_rows);
  s.lq = seq_rows(p.q_off, b, p.q_rows);
  s.k0 = clamp_int(p.k_off[b], 0, p.k_rows);
  s.lk = seq_rows(p.k_off, b, p.k_rows);
  if (p.k_len) s.lk = clamp_int(p.k_len[b], 0, s.lk);
  s.shift = s.lk - s.lq;
  s.prefix = p.prefix ? clamp_int(p.prefix[b], 0, s.lk) : 0;
  return s;
}

// Finds, with the 32 lanes of one warp, the sequence and the tile in it that tile number `tile` stands for when every
// sequence has ceil(rows / tile_rows) tiles; false behind the last one.  A sequence's tiles count from its end: under
// a causal mask the last rows have the most keys, and long work that starts first ends with the rest.
__device__ __forceinline__ bool find_tile(const int32_t* off, int n_seqs, int rows, int tile_rows, int tile, int* seq,
                                          int* index) {
  const int lane = threadIdx.x & 31;
  for (int base = 0; base < n_seqs; base += 32) {
    const int b = base + lane;
    const int n = b < n_seqs ? (seq_rows(off, b, rows) + tile_rows - 1) / tile_rows : 0;
    int sum = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += up;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, tile < sum);
    if (hit) {
      const int l = __ffs(hit) - 1;
      const int end = __shfl_sync(0xffffffffu, sum, l);
      *seq = base + l;
      *index = end - 1 - tile;
      return true;
    }
    tile -= __shfl_sync(0xffffffffu, sum, 31);
  }
  return false;
}

// Keys that a query at position `pos` sees: [lo, hi) and everything before `prefix`.
struct RowKeys {
  int lo, hi, prefix;
  __device__ __forceinline__ bool sees(int j) const { return (j >= lo && j < hi) || j < prefix; }
};
__device__ __forceinline__ RowKeys row_keys(const AttnSeq& s, int causal, int window, int pos) {
  RowKeys r{0, s.lk, s.prefix};
  if (causal) r.hi = min(r.hi, pos + 1);
  if (window) {
    r.lo = max(0, pos - window + 1);
    r.hi = (int)min((long long)r.hi, (long long)pos + window);
  }
  return r;
}

// Key tiles (of TILE keys) that the queries at positions [p0, p1] need: tiles [0, pre) and [lo, hi), pre <= lo.
template <int TILE>
struct KeyTiles {
  int pre, lo, hi;
  __device__ __forceinline__ int count() const { return pre + max(hi - lo, 0); }
  __device__ __forceinline__ int at(int i) const { return i < pre ? i : lo + i - pre; }
  __device__ __forceinline__ bool has(int t) const { return t < pre || (t >= lo && t < hi); }
};
template <int TILE>
__device__ __forceinline__ KeyTiles<TILE> key_tiles(const AttnSeq& s, int causal, int window, int p0, int p1) {
  KeyTiles<TILE> t;
  const int first = row_keys(s, causal, window, p0).lo, last = max(row_keys(s, causal, window, p1).hi, s.prefix);
  t.lo = min(first, s.lk) / TILE;
  t.hi = (max(last, 0) + TILE - 1) / TILE;
  t.pre = min((s.prefix + TILE - 1) / TILE, t.lo);
  return t;
}

// Query rows [lo, hi) that may see one of the keys [j0, j1).
__device__ __forceinline__ void query_rows(const AttnSeq& s, int causal, int window, int j0, int j1, int* lo, int* hi) {
  *lo = 0;
  *hi = s.lq;
  if (j0 < s.prefix) return;
  if (causal) *lo = clamp_int(j0 - s.shift, 0, s.lq);
  if (window) {
    if (!causal) *lo = (int)max((long long)*lo, min((long long)s.lq, (long long)j0 - s.shift - window + 1));
    *hi = (int)max((long long)*lo, min((long long)s.lq, (long long)j1 - 1 - s.shift + window));
  }
}

// Bits 0 to n - 1, of 32
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : (1u << max(n, 0)) - 1u; }
// Of 32 keys from j0: those that `lo`, `hi` and `prefix`, counted from j0, leave visible
__device__ __forceinline__ uint32_t seen_bits(int lo, int hi, int prefix) {
  return (low_bits(hi) & ~low_bits(lo)) | low_bits(prefix);
}

// 2^x in one special-function operation (within 2^-22 of the value; below 2^-126 it gives zero)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The two values of a bf16 pair
__device__ __forceinline__ float bf16_lo(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }
// Two fp32 values to an instruction
__device__ __forceinline__ uint64_t pair2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair2(uint64_t p, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  const __nv_bfloat162 e = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&e);
}

// A block's walk over (tile, head) pairs: rounds over the sorted tiles with the heads fastest, every other round from
// the other end.  One 32-byte load tells a tile; the next one is fetched while this one is worked on.
struct TileWalk {
  const AttnTile* table;
  int items, heads, round;
  int4 ahead[2];
  AttnSeq sq;
  int row0, head;
  __device__ __forceinline__ int item(int r) const {
    return r * (int)gridDim.x + ((r & 1) ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x);
  }
  __device__ __forceinline__ void fetch(int r) {
    const long long i = (long long)r * gridDim.x < items ? item(r) : items;
    if (i < items) {
      const int4* src = reinterpret_cast<const int4*>(table + i / heads);
      ahead[0] = src[0];
      ahead[1] = src[1];
    }
  }
  __device__ __forceinline__ TileWalk(const AttnTile* t, const int32_t* n, int h)
      : table(t), items(*n * h), heads(h), round(0) { fetch(0); }
  __device__ __forceinline__ bool next() {
    if ((long long)round * gridDim.x >= items) return false;
    const int i = item(round);
    if (i >= items) {                            // a gap of the last, partial round
      ++round;
      return false;
    }
    sq = AttnSeq{ahead[0].x, ahead[0].y, ahead[0].z, ahead[0].w, ahead[1].x, ahead[1].y};
    row0 = ahead[1].z;
    head = i % heads;
    fetch(++round);
    return true;
  }
};

// tanh from two special-function operations: 1 - 2 / (1 + e^(2x)).  Its absolute error is a few 2^-24.
__device__ __forceinline__ float tanh_fast(float x) {
  return 1.f - __fdividef(2.f, 1.f + ex2(x * (2.f * kLog2e)));
}

// Up to 3/4 tanh is taken on the fp32 pipes: the odd polynomial of degree 11 with the least absolute error there (7e-8 in
// fp32; fitted for this purpose by linear programming; 2.6e-7 of the value, so that scores far below a large cap keep
// theirs).  2.5 times as fast as two special-function operations a value.
constexpr float kTanhPoly = 0.75f;
__device__ __forceinline__ uint64_t tanh_poly(uint64_t u) {
  const uint64_t t = mul2(u, u);
  uint64_t y = fma2(t, pair2(-0.004493420943617821f, -0.004493420943617821f), pair2(0.019237183034420013f, 0.019237183034420013f));
  y = fma2(y, t, pair2(-0.053149230778217316f, -0.053149230778217316f));
  y = fma2(y, t, pair2(0.13320578634738922f, 0.13320578634738922f));
  y = fma2(y, t, pair2(-0.33332470059394836f, -0.33332470059394836f));
  y = fma2(y, t, pair2(0.9999998211860657f, 0.9999998211860657f));
  return mul2(y, u);
}

__device__ __forceinline__ float tanh_one(float x) {
  float p, unused;
  unpair2(tanh_poly(pair2(x, 0.f)), p, unused);
  return fabsf(x) > kTanhPoly ? tanh_fast(x) : p;
}

// x <- tanh(x * mul) for a thread's scores.  What a value becomes depends on itself alone: the values of a warp only decide
// together whether any of them needs the special functions, so hidden keys and rows of other sequences change nothing.
// Where one does the warp computes both forms of every value (4096 rows, 16 heads of 128: forward 86 us without any, 119
// with; 110 with the special functions alone).
template <int N>
__device__ __forceinline__ void tanh_all(float (&x)[N], float mul) {
  float mx[2] = {0.f, 0.f};
#pragma unroll
  for (int j = 0; j < N; ++j) mx[j & 1] = fmaxf(mx[j & 1], fabsf(x[j]));
  if (__any_sync(0xffffffffu, fmaxf(mx[0], mx[1]) * mul > kTanhPoly)) {
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      float u0, u1, p0, p1;
      const uint64_t u = mul2(pair2(x[j], x[j + 1]), pair2(mul, mul));
      unpair2(u, u0, u1);
      unpair2(tanh_poly(u), p0, p1);
      const float f0 = tanh_fast(u0), f1 = tanh_fast(u1);
      x[j] = fabsf(u0) > kTanhPoly ? f0 : p0;
      x[j + 1] = fabsf(u1) > kTanhPoly ? f1 : p1;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 2)
      unpair2(tanh_poly(mul2(pair2(x[j], x[j + 1]), pair2(mul, mul))), x[j], x[j + 1]);
  }
}

// Lets a kernel use `bytes` of dynamic shared memory: asked of the runtime once per kernel and device.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, bool (&done)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev >= 0 && dev < 64 && done[dev])) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;      // a race only repeats the call
  return e;
}

// Launches of one call follow each other closely: a kernel launched with launch_behind() may start, and set itself up, as
// soon as every block of the kernel before it has begun (let_next_start), and waits for that kernel's end and results
// with wait_for_last before it touches anything that the call's kernels share.  Saves 2 to 3 us a launch.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... Params, typename... Args>
cudaError_t launch_behind(void (*kernel)(Params...), unsigned grid, unsigned block, size_t smem, cudaStream_t st,
                          const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

// Plans the tiles of `tile_rows` query rows (keys: of keys): `table` of `capacity` entries, `first` [n_seqs] scratch.  Also
// clears the status word.
struct AttnPlanJob {
  AttnTile* table;
  int32_t *count, *first;
  int tile_rows, capacity, keys;
};
cudaError_t launch_attn_plan(const AttnArgs& p, const AttnPlanJob* jobs, int n_jobs, cudaStream_t st);
int attn_sm_count();
constexpr int kFwdTile = 256, kBwdTile = 128;

cudaError_t launch_attn_forward_tc(const AttnArgs& p, cudaStream_t st);
cudaError_t launch_attn_backward_tc(const AttnArgs& p, cudaStream_t st);
cudaError_t launch_attn_forward_simt(const AttnArgs& p, cudaStream_t st);
cudaError_t launch_attn_backward_simt(const AttnArgs& p, cudaStream_t st);
cudaError_t launch_attn_delta(const AttnArgs& p, bool bf16_mode, float* lse2, float* delta, cudaStream_t st);

// Few query rows for each sequence and key head: a split over the keys, joined by a second launch.
constexpr int kFewRows = 16;                     // rows of a block
constexpr int kFewRowsMax = 64;                  // rows of a sequence and key head up to which this form is taken
struct FewSplits { int count; bool cluster; };   // more than one without a cluster: partials in the workspace
FewSplits attn_few_splits(int n_seqs, int kv_heads, int rows, long long k_rows, int max_k_len);
cudaError_t launch_attn_few(const AttnArgs& p, bool bf16_mode, FewSplits splits, float* part, cudaStream_t st);

}  // namespace mixlora
