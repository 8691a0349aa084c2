// The tiles of a packed batch, longest work first, for the persistent attention kernels.
//
// One block per table.  A sequence's tiles are counted and summed up over the sequences, every tile is given its work (the
// number of tiles of the other side that it meets), and a counting sort by work, largest first, writes the table.  The
// main kernels deal it out to their blocks in turn, forwards and backwards, so that blocks end together although causal
// rows and ragged sequences make the tiles' work differ by any factor.  The order among tiles of equal work may differ
// from call to call; no result depends on it.  3.5 us at a few dozen sequences, most of it latency.
#include "attention.cuh"

namespace mixlora {
namespace {

constexpr int kThreads = 1024;
constexpr int kLevels = 1024;                    // works from kLevels - 1 on are not told apart

// Inclusive sum over the block; `total` gets the sum of all.
__device__ __forceinline__ int block_sum(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += up;
  }
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  if (warp == 0) {
    int s = warp_sums[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += up;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  if (warp > 0) v += warp_sums[warp - 1];
  *total = warp_sums[31];
  __syncthreads();
  return v;
}

__global__ void __launch_bounds__(kThreads) attn_plan_kernel(AttnArgs a, AttnPlanJob job0, AttnPlanJob job1) {
  let_next_start();
  const AttnPlanJob job = blockIdx.x == 0 ? job0 : job1;
  __shared__ int warp_sums[32], levels[kLevels], first_near[kThreads];
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) *a.status = 0;
  for (int i = threadIdx.x; i < kLevels; i += kThreads) levels[i] = 0;
  int total = 0;
  for (int b0 = 0; b0 < a.n_seqs; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int n = 0;
    if (b < a.n_seqs) {
      const AttnSeq s = load_seq(a, b);
      n = ((job.keys ? s.lk : s.lq) + job.tile_rows - 1) / job.tile_rows;
    }
    int sum;
    const int upto = block_sum(n, warp_sums, &sum);
    if (b < a.n_seqs) {
      job.first[b] = total + upto - n;
      if (b0 == 0) first_near[b] = upto - n;
    }
    total += sum;
  }
  __syncthreads();                               // `first` is read by other threads of this block
  const int* first = a.n_seqs <= kThreads ? first_near : job.first;
  total = min(total, job.capacity);              // offsets that overlap could ask for more
  // the tile with number i: its sequence is the last one that starts at or before it and has tiles
  auto tile = [&](int i, AttnTile* t) {
    int lo = 0, hi = a.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    t->sq = load_seq(a, lo);
    t->row0 = (i - first[lo]) * job.tile_rows;
    const AttnSeq& s = t->sq;
    int work;
    if (job.keys) {
      int r0, r1;
      query_rows(s, a.causal, a.window, t->row0, min(t->row0 + job.tile_rows, s.lk), &r0, &r1);
      work = (max(r1 - r0, 0) + 127) / 128;
    } else {
      const int last = min(t->row0 + job.tile_rows, s.lq) - 1;
      work = key_tiles<128>(s, a.causal, a.window, s.shift + t->row0, s.shift + last).count();
    }
    return kLevels - 1 - min(work, kLevels - 1);
  };
  AttnTile t;                                    // a thread's first tile is kept for the second pass
  int level = 0;
  if ((int)threadIdx.x < total) {
    level = tile(threadIdx.x, &t);
    atomicAdd(&levels[level], 1);
  }
  for (int i = threadIdx.x + kThreads; i < total; i += kThreads) {
    AttnTile u;
    atomicAdd(&levels[tile(i, &u)], 1);
  }
  __syncthreads();
  int sum;
  const int mine = levels[threadIdx.x], upto = block_sum(mine, warp_sums, &sum);
  levels[threadIdx.x] = upto - mine;
  __syncthreads();
  for (int i = threadIdx.x; i < total; i += kThreads) {
    if (i >= kThreads) level = tile(i, &t);
    const int at = atomicAdd(&levels[level], 1);
    int4* dst = reinterpret_cast<int4*>(job.table + at);
    dst[0] = make_int4(t.sq.q0, t.sq.lq, t.sq.k0, t.sq.lk);
    dst[1] = make_int4(t.sq.shift, t.sq.prefix, t.row0, 0);
  }
  if (threadIdx.x == 0) *job.count = total;
}

}  // namespace

cudaError_t launch_attn_plan(const AttnArgs& a, const AttnPlanJob* jobs, int n_jobs, cudaStream_t st) {
  attn_plan_kernel<<<n_jobs, kThreads, 0, st>>>(a, jobs[0], jobs[n_jobs - 1]);
  return cudaGetLastError();
}

int attn_sm_count() {
  static int sms[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if (sms[dev] == 0) {
    int n = 0;
    sms[dev] = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0 ? n : 148;
  }
  return sms[dev];
}

}  // namespace mixlora
