// What the head's losses do once a row: which rows count, a teacher's lists, and the join of a row's tiles.
//
// All of it is small beside the products (8192 rows of 32000 columns: scan 9, join 27 of 3410 us; 4096 rows with 64 entries:
// lists 10, scan 6, rows side by side 10, join 30 of 1670), so what can lose bits by cancellation is done in 64 bits:
// probabilities of a teacher, log-sum-exps, gradients towards listed columns.  With few rows these kernels wait for one load
// after another; each starts under its predecessor, and the join is 5 to 9 us of a call of 40.
#include <math.h>
#include <string.h>

#include "head.cuh"

namespace mixlora {
namespace {

constexpr double kLn2d = 0.69314718055994530942, kLog2ed = 1.44269504088896340736;
constexpr int kListThreads = 128;
constexpr int kScanThreads = 1024, kScanEach = 8;
constexpr int kRowThreads = 32 * kHeadRowsPerBlock;

template <typename T> __device__ __forceinline__ T warp_sum(T v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}

constexpr int kCopies = 4;      // 16-byte loads that a lane has under way
// A row of n fp32 values (a multiple of 8) into three rows of bf16, `apart` values from one to the next, by a warp
__device__ __forceinline__ void take_apart(const float* src, bf16* dst, size_t apart, int n) {
  for (int i0 = (threadIdx.x & 31) * 4; i0 < n; i0 += 128 * kCopies) {
    float4 v[kCopies];
#pragma unroll
    for (int j = 0; j < kCopies; ++j)
      if (i0 + 128 * j < n) v[j] = *reinterpret_cast<const float4*>(src + i0 + 128 * j);
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
      if (i0 + 128 * j >= n) break;
      const HeadParts a = head_parts(v[j].x), b = head_parts(v[j].y), c = head_parts(v[j].z), d = head_parts(v[j].w);
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(a.v[k], b.v[k]), up = __floats2bfloat162_rn(c.v[k], d.v[k]);
        *reinterpret_cast<uint2*>(dst + k * apart + i0 + 128 * j) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&up));
      }
    }
  }
}

// A teacher's entries of one token, a warp each: columns ascending, an entry outside the vocabulary dropped, entries of the
// same column added up; their probabilities and what they leave over.  An entry's place is the number of entries before
// it, counted by comparing it with all (at most 256 x 256 / 32 steps of a warp).
__global__ void __launch_bounds__(kListThreads) head_lists_kernel(HeadArgs p) {
  let_next_start();
  extern __shared__ char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * (kListThreads / 32) + warp;
  if (t >= p.tokens) return;
  const int top = p.top, each = (top + 31) / 32;
  double* prob = reinterpret_cast<double*>(smem) + (size_t)warp * 2 * top;      // by entry, then by place
  int* col = reinterpret_cast<int*>(reinterpret_cast<double*>(smem) + (size_t)(kListThreads / 32) * 2 * top) + (size_t)warp * 2 * top;
  const int32_t* index = p.t_index + (size_t)t * top;
  const float* logit = p.t_logit + (size_t)t * top;
  double most = -INFINITY;
  for (int k = lane; k < top; k += 32) {
    const int c = index[k];
    const bool in = c >= 0 && c < p.vocab;
    col[k] = in ? c : kHeadNone;
    const double z = (double)logit[k] / (double)p.temperature;
    prob[k] = z;
    if (in) most = fmax(most, z);
  }
  most = warp_max(most);
  const bool whole = p.t_lse != nullptr;
  // without the teacher's sum a list of nothing but -inf says nothing; with it, it says that these are not chosen
  const double from = whole ? (double)p.t_lse[t] : most;
  __syncwarp();
  for (int k = lane; k < top; k += 32) {
    const int c = col[k];
    int place = 0;
    for (int j = 0; j < top; ++j) place += col[j] < c || (col[j] == c && j < k);
    col[top + place] = c;
    prob[top + place] = c == kHeadNone || (most == -INFINITY && !isnan(prob[k])) ? 0.0 : exp(prob[k] - from);
  }
  __syncwarp();
  // first entries of their column, in order: 32 places at a time
  double sum = 0.0;
  int n = 0;
  for (int i = 0; i < each; ++i) {
    const int k = i * 32 + lane;
    const int c = k < top ? col[top + k] : kHeadNone;
    const bool lead = c != kHeadNone && (k == 0 || col[top + k - 1] != c);
    double q = 0.0;
    if (lead)
      for (int j = k; j < top && col[top + j] == c; ++j) q += prob[top + j];
    const unsigned leads = __ballot_sync(0xffffffffu, lead);
    const int at = n + __popc(leads & ((1u << lane) - 1u));
    if (lead) {
      col[at] = c;              // at <= k: that place has been read, col[.. top) is free since the sort
      prob[at] = q;
    }
    sum += lead ? q : 0.0;
    n += __popc(leads);
  }
  sum = warp_sum(sum);
  __syncwarp();
  if (!whole && sum == 0.0) n = 0;
  for (int k = lane; k < top; k += 32) {
    p.list_out[(size_t)t * top + k] = k < n ? col[k] : kHeadNone;
    p.list_q[(size_t)t * top + k] = k < n ? (whole ? prob[k] : prob[k] / sum) : 0.0;
  }
  if (lane == 0) {
    p.list_n[t] = n;
    // a list of every column leaves nothing over, whatever its sum was rounded to; a sum that is no number says so
    p.rest_q[t] = whole && n < p.vocab ? (sum >= 1.0 ? 0.0 : 1.0 - sum) : 0.0;
  }
}

// What a weight is multiplied by: one over the normalizer, in 64 bits, where that of the smallest fp32 weights has a value
__device__ __forceinline__ double part_of_each(const HeadArgs& p, double weights) {
  const double norm = p.normalizer ? (double)p.normalizer[0] : weights;
  return norm == 0.0 ? 0.0 : 1.0 / norm;
}

// Numbers the counted rows and adds up their weights: one block, 8192 tokens a turn, eight to a thread and a warp's 32 side
// by side.  Rows that are left out get their zeroes here.
__global__ void __launch_bounds__(kScanThreads) head_scan_kernel(HeadArgs p) {
  constexpr int kWarps = kScanThreads / 32, kCounts = kScanEach * kWarps;
  let_next_start();
  wait_for_last();
  __shared__ int counts[kCounts], of_eight[32];            // counted tokens of each 32, then of those before them
  __shared__ double warp_w[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int base = 0;
  double weight = 0.0;
  for (int t0 = 0; t0 < p.tokens; t0 += kScanThreads * kScanEach) {
    unsigned in[kScanEach];
#pragma unroll
    for (int j = 0; j < kScanEach; ++j) {
      const int t = t0 + j * kScanThreads + threadIdx.x;
      const bool ok = t < p.tokens && head_entries(p, t) > 0;
      in[j] = __ballot_sync(0xffffffffu, ok);
      if (ok) {
        weight += p.weights ? (double)p.weights[t] : 1.0;
      } else if (t < p.tokens) {
        p.loss[t] = 0.f;
        if (p.lse) p.lse[t] = 0.f;
      }
      if (lane == 0) counts[j * kWarps + warp] = __popc(in[j]);
    }
    __syncthreads();
    // 256 counts: 32 threads add up eight each, and one of those 32
    if (threadIdx.x < kCounts / 8) {
      int sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int n = counts[threadIdx.x * 8 + j];
        counts[threadIdx.x * 8 + j] = sum;
        sum += n;
      }
      int upto = sum;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += up;
      }
      of_eight[lane] = upto;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kScanEach; ++j) {
      const int t = t0 + j * kScanThreads + threadIdx.x, at = j * kWarps + warp;
      if (t >= p.tokens) continue;
      const int row = base + counts[at] + (at >= 8 ? of_eight[at / 8 - 1] : 0) + __popc(in[j] & ((1u << lane) - 1u));
      const bool ok = in[j] >> lane & 1;
      p.token_row[t] = ok ? row : -1;
      if (ok) p.row_token[row] = t;
    }
    base += of_eight[31];
    __syncthreads();
  }
  weight = warp_sum(weight);
  if (lane == 0) warp_w[warp] = weight;
  __syncthreads();
  if (threadIdx.x == 0) {
    double sum = 0.0;
    for (int i = 0; i < kWarps; ++i) sum += warp_w[i];
    p.state->status = 0;
    p.state->counted = base;
    p.state->joined = 0;
    p.state->weight = (float)sum;
    p.state->each = part_of_each(p, sum);
  }
}
static_assert(kScanEach * kScanThreads / 32 == 256, "the scan's counts are added up by one warp, eight a lane");

// The counted rows of this piece side by side, where tokens are left out (the products then pass over nothing else) or an
// fp32 row is taken apart.  A warp a token before the first piece, whose launch also writes zeroes for the gradients of the tokens
// that are left out, and a warp a row of the piece before the others (2^20 tokens of 4096 columns, width 64, half of them left
// out, 8 pieces and 8 without rows: 8.3 -> 6.8 ms).
template <int PARTS>
__global__ void __launch_bounds__(kRowThreads) head_gather_kernel(HeadArgs p) {
  let_next_start();
  wait_for_last();
  if (PARTS == 1 && p.state->counted == p.tokens) return;
  const int lane = threadIdx.x & 31;
  int t = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5), row = t;
  if (p.piece0 == 0) {
    if (t >= p.tokens) return;
    row = p.token_row[t];
  } else {
    if (row >= head_rows_here(p)) return;
    t = p.row_token[p.piece0 + row];
  }
  if (row < 0) {
    if (!p.d_x) return;
    constexpr int kEach = PARTS == 1 ? 8 : 4;              // values of 16 bytes
    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<char*>(p.d_x) + (size_t)t * p.dx_stride * (16 / kEach));
    for (int i = lane; i < p.d / kEach; i += 32) dst[i] = make_uint4(0, 0, 0, 0);
    return;
  }
  if (row >= p.piece) return;
  if (PARTS == 1) {
    const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(p.x) + (size_t)t * p.x_stride);
    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(p.x_rows) + (size_t)row * p.d);
    for (int i = lane; i < p.d / 8; i += 32 * kCopies) {
      uint4 v[kCopies];
#pragma unroll
      for (int j = 0; j < kCopies; ++j)
        if (i + 32 * j < p.d / 8) v[j] = src[i + 32 * j];
#pragma unroll
      for (int j = 0; j < kCopies; ++j)
        if (i + 32 * j < p.d / 8) dst[i + 32 * j] = v[j];
    }
  } else {
    take_apart(reinterpret_cast<const float*>(p.x) + (size_t)t * p.x_stride,
               reinterpret_cast<bf16*>(p.x_rows) + (size_t)row * p.d, (size_t)p.piece * p.d, p.d);
  }
}

// The head in parts, a warp a row: memory's 10 bytes a value; behind it, where rows are tokens, those of x.  It runs beside
// the scan or the lists, of which it needs nothing.
__global__ void __launch_bounds__(kRowThreads) head_parts_kernel(HeadArgs p) {
  let_next_start();
  const int row = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (row < p.vocab)
    take_apart(reinterpret_cast<const float*>(p.w) + (size_t)row * p.w_stride, p.w_parts + (size_t)row * p.d,
               (size_t)p.vocab * p.d, p.d);
  else if (p.few && row - p.vocab < p.tokens)
    take_apart(reinterpret_cast<const float*>(p.x) + (size_t)(row - p.vocab) * p.x_stride,
               reinterpret_cast<bf16*>(p.x_rows) + (size_t)(row - p.vocab) * p.d, (size_t)p.piece * p.d, p.d);
  wait_for_last();
}

// What a row needs of the exponential and the logarithm in 64 bits, good to 2^-32: a divergence is a small difference
// of logarithms.  Powers of two go by the exponent's bits, the rest by the series.  The library's functions are several times
// the code, and fetching that once a launch took longer than all of a row's work.
__device__ __forceinline__ double recip64(double x) {      // x in fp32's range
  double r = (double)__fdividef(1.f, (float)x);
  r = r * fma(-x, r, 2.0);
  return r * fma(-x, r, 2.0);
}
__device__ __forceinline__ double exp64(double x) {
  if (x < -690.0) return 0.0;
  const double k = rint(fmin(x, 700.0) * kLog2ed), t = fma(-k, kLn2d, x);      // |t| <= 0.35
  double y = 1.0 / 362880;                                 // t^n / n! up to the ninth: relatively, the tenth is 1e-11
  y = fma(y, t, 1.0 / 40320);
  y = fma(y, t, 1.0 / 5040);
  y = fma(y, t, 1.0 / 720);
  y = fma(y, t, 1.0 / 120);
  y = fma(y, t, 1.0 / 24);
  y = fma(y, t, 1.0 / 6);
  y = fma(y, t, 0.5);
  y = fma(y, t, 1.0);
  y = fma(y, t, 1.0);
  return y * __hiloint2double((1023 + (int)k) << 20, 0);
}
// ln((1 + t) / (1 - t)) = 2 (t + t^3 / 3 + ...), |t| <= 1/3: relatively, what is left out is 1e-10
__device__ __forceinline__ double twice_artanh(double t) {
  const double u = t * t;
  double y = 1.0 / 17;
#pragma unroll
  for (int n = 15; n >= 1; n -= 2) y = fma(y, u, 1.0 / n);
  return 2.0 * t * y;
}
__device__ __forceinline__ double log64(double x) {        // x > 0, or no number of either sign
  if (!(x <= 0x1.fffffffffffffp+1023)) return x;
  if (x < 0x1p-1000) x = 0x1p-1000;
  const int hi = __double2hiint(x);
  double m = __hiloint2double((hi & 0x000fffff) | 0x3ff00000, __double2loint(x));
  int e = (hi >> 20) - 1023;
  if (m > 1.4142135623730951) { m *= 0.5; ++e; }
  return twice_artanh((m - 1.0) * recip64(m + 1.0)) + e * kLn2d;
}
__device__ __forceinline__ double log1p64(double x) { return twice_artanh(x * recip64(2.0 + x)); }      // 0 <= x <= 1

// What a warp of the joining kernel works on
struct RowJob {
  const float2* stats;          // the row's tiles
  int tiles, n;                 // n: listed columns
  const int32_t* list;
  const double* q;              // the teacher's probabilities, or NULL: a label
  double rest, weight, each;
  float* z;                     // the listed logits; gets the places' values G_k / A
  float *loss, *lse, *scale;    // lse, scale: or NULL
  bf16* e;
  long long e_part;
};

// One row's loss and, with a gradient, what its columns need, by one warp.  The columns that are not listed come as
// s 2^r (s = 0: there is none).
struct RowResult { double r, weighted; };
__device__ __forceinline__ RowResult finish_row(const HeadArgs& p, const RowJob& job, double s, double r) {
  const int lane = threadIdx.x & 31, n = job.n;
  const double lr = s == 0.0 ? -INFINITY : r * kLn2d + log64(s);
  const double zeta = (double)p.z_loss;
  double loss, lse, most, miss = 0.0, mass = 1.0;
  const double* q = job.q;
  float* z = job.z;
  const double rest = job.rest;
  if (!q) {
    // loss = ln(1 + e^gap) without a difference of two logarithms, and 1 - p without one from one
    most = (double)__shfl_sync(0xffffffffu, lane == 0 ? z[0] : 0.f, 0);     // lane 0 writes it below
    const double gap = lr - most, e = exp64(-fabs(gap));
    loss = (gap < 0.0 ? 0.0 : gap) + log1p64(e);
    miss = (gap > 0.0 ? 1.0 : e) * recip64(1.0 + e);
    lse = most + loss;
  } else {
    most = -INFINITY;
    for (int k = lane; k < n; k += 32) most = fmax(most, (double)z[k]);
    most = warp_max(most);
    const double from = fmax(most, lr);
    double sum = 0.0;
    for (int k = lane; k < n; k += 32) sum += exp64((double)z[k] - from);
    sum = warp_sum(sum) + exp64(lr - from);
    lse = from + log64(sum);
    loss = mass = 0.0;
    for (int k = lane; k < n; k += 32) {
      mass += q[k];
      if (!(q[k] == 0.0)) loss += q[k] * (log64(q[k]) - ((double)z[k] - lse));
    }
    loss = warp_sum(loss);
    // what the target sums up to: 1 but where a teacher's entries exceed it, or name every column and stay below
    mass = warp_sum(mass) + rest;
    if (!(rest == 0.0)) loss += rest * (log64(rest) - (lr - lse));
  }
  loss += zeta * lse * lse;
  if (lane == 0) {
    *job.loss = (float)loss;
    if (job.lse) *job.lse = (float)lse;
  }
  RowResult out{r, job.weight * (double)(float)loss};
  if (!job.scale) return out;
  // The others' R, unless G_k / A could leave bf16's range there: then the next one that brings u above 2^-50.  What is left
  // over keeps the others' where it counts, since the whole of it goes into their E, however small they are
  if (s == 0.0) out.r = 100.0 * rint(most * (kLog2ed / 100.0));
  double u = exp64(out.r * kLn2d - lse), part = rest > 0.0 && s > 0.0 ? rest * recip64(s) : 0.0;
  if (s != 0.0 && fmax(u, part) < 0x1p-50) {
    out.r = r + 100.0 * ceil((lse * kLog2ed - r - 50.0) * 0.01);
    u = exp64(out.r * kLn2d - lse);
    const double s_row = exp64(lr - out.r * kLn2d);
    part = rest > 0.0 && s_row > 0x1p-100 ? rest * recip64(s_row) : 0.0;
  }
  const double curl = 2.0 * zeta * lse, share = mass + curl;
  double a = share * u - part;
  // nothing below what the 32-bit sums behind u and s can tell from zero, so that G_k / A stays in range
  const double least = 0x1p-30 * fmax(u, part);
  if (fabs(a) < least) a = a < 0.0 ? -least : least;
  double largest = 0.0;
  for (int k = lane; k < n; k += 32) {
    const double zk = (double)z[k], pk = exp64(zk - lse);
    double g = q ? share * pk - q[k] : curl * pk - miss;
    if (p.softcap > 0.f) {
      const double tk = zk * p.z_to_cap;
      g *= (1.0 - tk) * (1.0 + tk);
    }
    z[k] = (float)g;
    if (fabs(g) > fabs(largest)) largest = (double)(float)g;
  }
  if (p.parts == 1) {
    // the largest listed factor, most of the gradient where the others' are spread out, is made one that rounding keeps: A
    // takes up the difference
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      const double other = __shfl_xor_sync(0xffffffffu, largest, d);
      if (fabs(other) > fabs(largest) || (fabs(other) == fabs(largest) && other > largest)) largest = other;
    }
    const double near = (double)__bfloat162float(__float2bfloat16((float)(largest * recip64(a))));
    if (fabs(near) > 0x1p-100 && fabs(near) < 0x1p120) a = largest * recip64(near);
  }
  const double over = recip64(a);
  for (int k = lane; k < n; k += 32) z[k] = (float)((double)z[k] * over);
  if (lane == 0) *job.scale = (float)(a * p.z_per_xw * job.weight * job.each);
  return out;
}

// Joins a row's tiles, a warp a row: sums over the tiles' R and S, the row's loss, and for a gradient its exponentials at one
// R with the listed columns' factors in their places.  A ninth warp adds up the blocks' weighted losses meanwhile: the block
// that comes last does so, in the blocks' order.
//
// The blocks that can be there early run through their code once on a row of their own making while the kernel before them
// still runs: the instructions have then been fetched when the sums arrive (a launch of few rows waited longer for its 8 KB
// of them than it computed).
struct BlankRow { float2 stats; double q; float z, loss, lse, scale; int32_t list; bf16 e; };
__global__ void __launch_bounds__(kRowThreads + 32) head_join_kernel(HeadArgs p) {
  constexpr int kWarps = kRowThreads / 32, kAhead = 8, kWarmBlocks = 3 * 148;
  let_next_start();
  __shared__ double warp_w[kWarps];
  __shared__ float weights;
  __shared__ BlankRow blank[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (warp == kWarps) {
    wait_for_last();
    // blocks that have rows, over all pieces; where none has, the first one is left to write the totals
    const int block = p.piece0 / kWarps + blockIdx.x, counted = p.few ? p.tokens : p.state->counted,
              blocks = max((counted + kWarps - 1) / kWarps, 1);
    __syncthreads();
    if (block >= blocks) return;
    int last = 0;
    if (lane == 0) {
      double mine = 0.0;
      for (int i = 0; i < kWarps; ++i) mine += warp_w[i];
      p.loss_part[block] = mine;
      __threadfence();
      last = atomicAdd(&p.state->joined, 1) == blocks - 1;
    }
    if (!__shfl_sync(0xffffffffu, last, 0) || !p.totals) return;
    __threadfence();
    double sum = 0.0;
#pragma unroll 8
    for (int i = lane; i < blocks; i += 32) sum += __ldcg(p.loss_part + i);
    sum = warp_sum(sum);
    if (lane == 0) {
      p.totals[0] = (float)sum;
      p.totals[1] = weights;
    }
    return;
  }
#pragma unroll 1
  for (int pass = blockIdx.x < kWarmBlocks ? 0 : 1; pass < 2; ++pass) {
    RowJob job;
    memset(&job, 0, sizeof(job));
    float2 ahead[kAhead];                              // a lane's first tiles, asked for before anything else
    auto ask = [&](int i0) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) ahead[j] = i0 + 32 * j < job.tiles ? job.stats[i0 + 32 * j] : make_float2(0.f, 0.f);
    };
    if (pass == 0) {
      BlankRow& b = blank[warp];
      if (lane == 0) {
        b.stats = make_float2(0.f, 1.f);
        b.q = 1.0;
        b.z = 0.f;
        b.list = 0;
      }
      __syncwarp();
      job.stats = &b.stats; job.tiles = 1; job.n = 1;
      job.list = &b.list; job.q = p.labels ? nullptr : &b.q;
      job.z = &b.z; job.loss = &b.loss; job.lse = &b.lse; job.scale = p.d_x ? &b.scale : nullptr;
      job.e = &b.e;
      ask(lane);
    } else {
      wait_for_last();
      const int row = blockIdx.x * kWarps + warp;
      job.stats = p.stats + (size_t)row * p.col_tiles; job.tiles = p.col_tiles;
      ask(lane);
      const int rows = head_rows_here(p);
      if (p.few) {                                     // no kernel has been over the tokens before
        double sum = 0.0;
        for (int t = lane; t < p.tokens; t += 32)
          if (head_entries(p, t) > 0) sum += p.weights ? (double)p.weights[t] : 1.0;
        sum = warp_sum(sum);
        if (threadIdx.x == 0) weights = (float)sum;
        job.each = part_of_each(p, sum);
      } else {
        if (threadIdx.x == 0) weights = p.state->weight;
        job.each = p.state->each;
      }
      int token = p.few ? row : (p.piece0 + row < p.tokens ? p.row_token[p.piece0 + row] : -1);      // asked for together
      if (row >= rows) token = -1;
      if (token >= 0) {
        job.n = p.labels && !p.few ? 1 : head_entries(p, token);
        job.list = p.list + (size_t)token * p.top;
        job.weight = p.weights ? (double)p.weights[token] : 1.0;
        if (!p.labels) {
          job.q = p.list_q + (size_t)token * p.top;
          job.rest = p.rest_q[token];
          if (job.n == 1 && job.rest == 0.0 && job.q[0] == 1.0) job.q = nullptr;      // one column takes all: a label
        }
        job.z = p.z_listed + (size_t)row * p.top;
        job.loss = p.loss + token;
        job.lse = p.lse ? p.lse + token : nullptr;
        job.scale = p.d_x ? p.row_scale + row : nullptr;
        job.e = reinterpret_cast<bf16*>(p.e) + (size_t)row * p.pitch; job.e_part = p.e_part;
        if (p.few && lane == 0) {
          p.row_token[token] = token;
          p.token_row[token] = job.n ? token : -1;
          if (job.n == 0) {
            *job.loss = 0.f;
            if (job.lse) *job.lse = 0.f;
            if (job.scale) *job.scale = 0.f;
          }
        }
      }
    }
    RowResult res{0.0, 0.0};
    if (job.n) {
      float r = -INFINITY, s = 0.f;
      auto add = [&](float r2, float s2) {           // a sum of nothing has no say in R
        const float most = s2 == 0.f ? r : (s == 0.f ? r2 : fmaxf(r, r2));
        s = (s == 0.f ? 0.f : s * exp2f(r - most)) + (s2 == 0.f ? 0.f : s2 * exp2f(r2 - most));
        r = most;
      };
      for (int i0 = lane;;) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) add(ahead[j].x, ahead[j].y);
        i0 += 32 * kAhead;
        if (i0 >= job.tiles) break;
        ask(i0);
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) {
        const float r2 = __shfl_xor_sync(0xffffffffu, r, d), s2 = __shfl_xor_sync(0xffffffffu, s, d);
        add(r2, s2);
      }
      res = finish_row(p, job, (double)s, (double)r);
    }
    if (pass == 1) {
      if (lane == 0) warp_w[warp] = res.weighted;
      __syncthreads();                                 // the ninth warp goes on
    }
    if (job.n && job.scale) {
      for (int i0 = 0; i0 < job.tiles; i0 += 32) {
        float by = 0.f;
        if (i0 + lane < job.tiles) {
          const float2 v = job.stats[i0 + lane];
          if (v.y != 0.f) by = v.x - (float)res.r;
        }
        unsigned todo = __ballot_sync(0xffffffffu, by < 0.f);
        while (todo) {
          const int l = __ffs(todo) - 1;
          todo &= todo - 1;
          const float f = exp2f(__shfl_sync(0xffffffffu, by, l));
          const int c = (i0 + l) * p.cols + lane * 4;
          if (lane * 4 >= p.cols || c >= p.pitch) continue;
          for (int k = 0; k < p.parts; ++k) {
            uint2* at = reinterpret_cast<uint2*>(job.e + k * job.e_part + c);
            uint2 v = *at;
            __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float2 w = __bfloat1622float2(h[j]);
              h[j] = __floats2bfloat162_rn(w.x * f, w.y * f);
            }
            *at = v;
          }
        }
        __syncwarp();
      }
      for (int k = lane; k < job.n; k += 32) {
        bf16* at = job.e + job.list[k];
        if (p.parts == 1) {
          *at = __float2bfloat16(job.z[k]);
        } else {
          const HeadParts v = head_parts(job.z[k]);
#pragma unroll
          for (int j = 0; j < 3; ++j) at[j * job.e_part] = __float2bfloat16(v.v[j]);
        }
      }
    }
  }
}

}  // namespace

cudaError_t launch_head_lists(const HeadArgs& p, cudaStream_t st) {
  constexpr int kWarps = kListThreads / 32;
  const size_t smem = (size_t)kWarps * 2 * p.top * (sizeof(double) + sizeof(int));   // 24 KB at 256 entries
  head_lists_kernel<<<(p.tokens + kWarps - 1) / kWarps, kListThreads, smem, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_head_scan(const HeadArgs& p, bool first, cudaStream_t st) {
  if (!first) return launch_behind(head_scan_kernel, 1, kScanThreads, 0, st, p);
  head_scan_kernel<<<1, kScanThreads, 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_head_parts(const HeadArgs& p, bool first, cudaStream_t st) {
  const int rows = p.vocab + (p.few ? p.tokens : 0);
  const unsigned blocks = (unsigned)((rows + kRowThreads / 32 - 1) / (kRowThreads / 32));
  if (!first) return launch_behind(head_parts_kernel, blocks, kRowThreads, 0, st, p);
  head_parts_kernel<<<blocks, kRowThreads, 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_head_gather(const HeadArgs& p, cudaStream_t st) {
  const int rows = p.piece0 == 0 ? p.tokens : p.piece;
  const unsigned blocks = (unsigned)((rows + kRowThreads / 32 - 1) / (kRowThreads / 32));
  return p.parts == 1 ? launch_behind(head_gather_kernel<1>, blocks, kRowThreads, 0, st, p)
                      : launch_behind(head_gather_kernel<3>, blocks, kRowThreads, 0, st, p);
}

cudaError_t launch_head_join(const HeadArgs& p, cudaStream_t st) {
  return launch_behind(head_join_kernel, (unsigned)((p.piece + kHeadRowsPerBlock - 1) / kHeadRowsPerBlock), kRowThreads + 32, 0,
                       st, p);
}

}  // namespace mixlora
