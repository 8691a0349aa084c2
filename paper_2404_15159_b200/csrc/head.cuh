// Shared parts of the losses on the output head: arguments, and how a row's exponentials are held.
//
// Logits z_v = (capped) scale x . w_v / temperature of a row are formed up to 128 columns at a time and turned into
// exponentials at once.  A row's `listed` columns (its label, or the teacher's entries) are left out of them and kept as
// fp32 logits: a sum or a difference that a confident row makes small is then never taken of nearly equal numbers, and is as good
// as the logits themselves.
//   those columns         R = 100 rint(log2(e) max z / 100) over its columns that are not listed, S = sum 2^(z log2(e) - R)
//   gradient              E_v = 2^(z_v log2(e) - R) (1 - (z_v temperature / softcap)^2), one rounding to bf16
// R is a multiple of 100, so tiles of a row nearly always share it, and where they do not (logits 35 apart or more) the
// row is brought to the largest one by powers of two, which round nothing.  With the row's R and
//   u = 2^R / sum e^z = p_v / E_v,    A = (1 + 2 z_loss lse) u - rest / S      (1: what the target sums up to)
// the gradient towards z_v is A E_v for a column that is not listed, and G_k for a listed one, which goes into the place
// of E as G_k / A: the gradient towards x is A times one product of E with w.
#pragma once

#include "common.cuh"
#include "launch.cuh"

namespace mixlora {

constexpr int kHeadTile = 256;               // rows and columns of a tile of the products
constexpr int kHeadCols = 128;               // most columns that share R and S
constexpr int kHeadLeastCols = 64;
constexpr float kHeadStep = 100.f;           // R's step, in powers of two
constexpr int kHeadFewTokens = 64;           // tokens up to which the head is streamed (bf16)
constexpr int kHeadNone = 0x7fffffff;        // no column (ends a row's list)
constexpr int kHeadMaxShares = 16;           // CTA pairs that share one tile's reduction
constexpr int kHeadMaxItems = 222;           // shares under way: three rounds of 74 CTA pairs
constexpr int kHeadPairs = 74;               // CTA pairs of a B200
constexpr int kHeadMostPairs = 128;          // CTA pairs that a launch uses at most
constexpr int kHeadRowsPerBlock = 8;         // rows that a block of the joining kernel takes

// What the kernels of a call leave for one another beside the arrays
struct HeadState {
  int32_t status;       // the device status word
  int32_t counted;      // rows with a label (an entry), the only ones that are computed
  int32_t joined;       // blocks of the joining kernel that are done
  float weight;         // sum of the counted rows' weights
  double each;          // 1 / normalizer
};

struct HeadArgs {
  const void *x, *w;              // [tokens, d], [vocab, d]
  void* d_x;                      // [tokens, d] or NULL
  long long x_stride, w_stride, dx_stride;
  int tokens, d, vocab, top;      // top: entries of a row's list (1 for labels)
  const int32_t* labels;          // [tokens], or NULL: a teacher's lists
  const int32_t* t_index;         // [tokens, top]
  const float *t_logit, *t_lse;   // [tokens, top], [tokens] or NULL
  const float *weights, *normalizer;   // or NULL
  float *loss, *lse, *totals;     // lse, totals: or NULL
  float scale, softcap, temperature, z_loss;
  double z_per_xw, z_to_cap;      // a logit for x . w where no cap bends it; a logit to what the cap's tanh gave
  float logit_factor;             // logits, before a cap, are this times x . w; a cap's are cap_out tanh(this times x . w)
  float cap_out, to2;             // to2: from x . w (from the tanh) to log2(e) times the logit
  // workspace
  HeadState* state;
  int32_t* row_token;             // [tokens] token of each counted row, ascending
  int32_t* token_row;             // [tokens] its inverse, -1 for a token that is left out
  const int32_t* list;            // [tokens, top] listed columns ascending, kHeadNone behind the last (labels: the labels)
  int32_t* list_out;              // the same, where it is made here
  double *list_q, *rest_q;        // [tokens, top], [tokens] teacher probabilities, and what they leave over
  int32_t* list_n;                // [tokens] entries, 0: left out
  double* loss_part;              // sum of weight * loss for each block of the joining kernel
  void* x_rows;                   // [parts, piece, d] the counted rows of x, where some tokens are left out or in parts
  bf16* w_parts;                  // [parts, vocab, d] fp32 mode: the head in parts
  float* z_listed;                // [piece, top] logits of the listed columns
  float2* stats;                  // [piece, col_tiles] (R, S)
  void* e;                        // [parts, piece, pitch]
  long long e_part;               // values from a part of E to the next
  float* row_scale;               // [piece]
  float* part;                    // partial tiles of a split reduction
  // the piece of counted rows that a launch works on
  int piece0, piece;              // first row, most rows
  int pitch, cols, col_tiles;     // cols: columns that share R and S, half a tile of the logits
  int part_items;                 // that `part` has room for
  int parts;                      // bf16 values that hold an operand: 1, or 3 in the fp32 mode
  int few;                        // no more tokens than a tile has rows: rows are tokens, those that are left out among them
};

// Entries of a token's list, 0 where it is left out
__device__ __forceinline__ int head_entries(const HeadArgs& p, int token) {
  return p.labels ? (p.labels[token] >= 0 && p.labels[token] < p.vocab) : p.list_n[token];
}
__device__ __forceinline__ int head_rows_here(const HeadArgs& p) {
  return p.few ? p.tokens : min(max(p.state->counted - p.piece0, 0), p.piece);
}
__device__ __forceinline__ int head_token(const HeadArgs& p, int row) { return p.few ? row : p.row_token[p.piece0 + row]; }
// Whether a token has no gradient, whatever its sums are
__device__ __forceinline__ bool head_left_out(const HeadArgs& p, int token) { return p.few && p.token_row[token] < 0; }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A value as the sum of three bf16 ones: the first is cut off (rounding could overflow), the others are rounded, which
// leaves nothing of 24 bits.
__device__ __forceinline__ float head_cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
struct HeadParts { float v[3]; };
__device__ __forceinline__ HeadParts head_parts(float x) {
  HeadParts p;
  p.v[0] = head_cut(x);
  const float rest = x - p.v[0];
  p.v[1] = __bfloat162float(__float2bfloat16(rest));
  p.v[2] = rest - p.v[1];
  return p;
}

cudaError_t launch_head_lists(const HeadArgs& p, cudaStream_t st);        // a teacher's entries: list, list_q, rest_q, list_n
cudaError_t launch_head_scan(const HeadArgs& p, bool first, cudaStream_t st);   // row_token, token_row, state (few tokens: none of it needed)
cudaError_t launch_head_parts(const HeadArgs& p, bool first, cudaStream_t st);   // fp32 mode: w_parts; x_rows where rows are tokens
cudaError_t launch_head_gather(const HeadArgs& p, cudaStream_t st);       // x_rows; before the first piece zeroes of d_x
cudaError_t launch_head_logits_tc(const HeadArgs& p, cudaStream_t st);    // stats, z_listed, E
cudaError_t launch_head_logits_few(const HeadArgs& p, bool first, cudaStream_t st);   // the same for up to kHeadFewTokens; clears the state
cudaError_t launch_head_join(const HeadArgs& p, cudaStream_t st);         // loss, lse, totals; E finished, row_scale
cudaError_t launch_head_grad_tc(const HeadArgs& p, cudaStream_t st);      // d_x
cudaError_t launch_head_grad_few(const HeadArgs& p, cudaStream_t st);
int head_few_shares(int d, int vocab);                                    // arrays [tokens, d] of it in `part`
int head_pairs();                                                         // CTA pairs of this GPU

}  // namespace mixlora
