// C ABI of the losses on the output head: argument checks, workspace layout, the launches piece by piece.
#include <math.h>
#include <string.h>

#include "head.cuh"

namespace mixlora {
namespace {

bool aligned(const void* p, size_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool aligned_or_null(const void* p, size_t n) { return !p || aligned(p, n); }

#define MIXLORA_TRY(expr)                               \
  do {                                                  \
    if ((expr) != cudaSuccess) return MIXLORA_ERR_CUDA; \
  } while (0)

// A stride as given or, for 0, dense; -1 if rows would overlap
long long stride_of(int64_t given, int width) { return given == 0 ? width : (given >= width ? (long long)given : -1); }

mixlora_status_t check_head(const mixlora_head_shape_t* s) {
  if (!s || s->struct_size != sizeof(mixlora_head_shape_t) || s->reserved != 0) return MIXLORA_ERR_INVALID_ARG;
  if (s->tokens < 0 || s->d_model <= 0 || s->vocab <= 0 || s->teacher_top < 0) return MIXLORA_ERR_INVALID_ARG;
  if (s->dtype != MIXLORA_DTYPE_BF16 && s->dtype != MIXLORA_DTYPE_FP32) return MIXLORA_ERR_INVALID_ARG;
  if (!isfinite(s->scale) || s->scale <= 0.f || !isfinite(s->temperature) || s->temperature <= 0.f ||
      !isfinite(s->softcap) || s->softcap < 0.f || !(s->z_loss >= 0.f && s->z_loss <= 0x1p20f))
    return MIXLORA_ERR_INVALID_ARG;
  // the factors that the kernels form of them, in fp32: none may leave the normal range
  if (!isnormal(s->scale / s->temperature) || !isnormal(s->scale / s->temperature * 1.4426950408889634f)) return MIXLORA_ERR_INVALID_ARG;
  if (s->softcap > 0.f && (!isnormal(s->scale / s->softcap) || !isnormal(s->softcap / s->temperature) ||
                           !isnormal(s->softcap / s->temperature * 1.4426950408889634f)))
    return MIXLORA_ERR_INVALID_ARG;
  const long long strides[] = {stride_of(s->x_stride, s->d_model), stride_of(s->w_stride, s->d_model),
                               stride_of(s->d_x_stride, s->d_model)};
  for (long long v : strides)
    if (v < 0) return MIXLORA_ERR_INVALID_ARG;
  if (s->d_model % 8 || s->d_model > 65536 || s->vocab > (1 << 20) || s->tokens > (1 << 24) ||
      s->teacher_top > MIXLORA_MAX_TEACHER_TOP)
    return MIXLORA_ERR_UNSUPPORTED;
  for (long long v : strides)
    if (v % 8 || v > (1LL << 32)) return MIXLORA_ERR_UNSUPPORTED;
  return MIXLORA_OK;
}

bool few_tokens(const mixlora_head_shape_t& s) { return s.dtype == MIXLORA_DTYPE_BF16 && s.tokens <= kHeadFewTokens; }

// Counted rows are worked on in pieces, as many as keep each of a piece's exponentials, rows of x and listed logits within 512
// MiB: enough for whole rounds of tiles, and the same whatever the batch.  Without a gradient there are two numbers for 128
// columns, and the copy of the rows of x is what counts.
int piece_rows(const mixlora_head_shape_t& s, bool gradient, int parts) {
  long long row = 2LL * parts * s.d_model;
  const long long wide = gradient ? 2LL * parts * s.vocab : (s.vocab + kHeadLeastCols - 1) / kHeadLeastCols * 8LL;
  if (row < wide) row = wide;
  if (row < 4LL * s.teacher_top) row = 4LL * s.teacher_top;          // the listed logits
  long long rows = (512LL << 20) / row / kHeadTile * kHeadTile;
  if (rows < kHeadTile) rows = kHeadTile;
  const long long all = ((long long)s.tokens + kHeadTile - 1) / kHeadTile * kHeadTile;
  return (int)(rows < all ? rows : (all > 0 ? all : kHeadTile));
}

// Columns of half a tile of the logits.  In fp32 mode, whose products outlast the way of their operands, a tile is made
// narrower where that fills the last round of CTA pairs better (700 tokens of 8009 columns 222 -> 203 us).  With bf16 a tile
// of 256 columns already waits for its operands: 512 tokens of 32000 columns take 4 rounds of 224 columns as long as 4 of 256.
int head_cols(const mixlora_head_shape_t& s, int parts, int piece) {
  if (parts == 1) return kHeadCols;
  const long long m_tiles = ((s.tokens < piece ? s.tokens : piece) + kHeadTile - 1) / kHeadTile;
  int best = kHeadCols;
  long long least = 0;
  for (int cols = kHeadCols; cols >= kHeadLeastCols; cols -= 16) {
    const long long tiles = m_tiles * ((s.vocab + 2 * cols - 1) / (2 * cols));
    const long long cost = (tiles + kHeadPairs - 1) / kHeadPairs * cols;
    if (cols == kHeadCols || cost < least) { least = cost; best = cols; }
  }
  return best;
}

struct HeadLayout {
  size_t state, row_token, token_row, list, list_q, rest_q, list_n, loss_part, x_rows, w_parts, z_listed, stats, e,
      row_scale, part, total;
  int parts, piece, pieces, pitch, cols, col_tiles, part_items;
};
HeadLayout head_layout(const mixlora_head_shape_t& s, bool gradient) {
  const size_t tokens = (size_t)s.tokens, top = s.teacher_top ? (size_t)s.teacher_top : 1;
  HeadLayout L;
  L.parts = s.dtype == MIXLORA_DTYPE_BF16 ? 1 : 3;
  L.piece = piece_rows(s, gradient, L.parts);
  L.pieces = (s.tokens + L.piece - 1) / L.piece;
  L.pitch = (s.vocab + 15) / 16 * 16;                      // rows of E start at 32 bytes
  L.cols = head_cols(s, L.parts, L.piece);
  L.col_tiles = (s.vocab + L.cols - 1) / L.cols;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
  L.state = take(sizeof(HeadState));
  L.row_token = take(tokens * 4);
  L.token_row = take(tokens * 4);
  const size_t lists = s.teacher_top ? tokens : 0;
  L.list = take(lists * top * 4);
  L.list_q = take(lists * top * 8);
  L.rest_q = take(lists * 8);
  L.list_n = take(lists * 4);
  L.loss_part = take((tokens / kHeadRowsPerBlock + 1) * 8);
  const size_t piece = (size_t)L.piece;
  L.x_rows = take(piece * s.d_model * 2 * L.parts);
  L.w_parts = take(L.parts == 3 ? (size_t)s.vocab * s.d_model * 6 : 0);
  L.z_listed = take(piece * top * 4);
  L.stats = take((size_t)L.col_tiles * piece * 8);
  L.e = take(gradient ? piece * L.pitch * 2 * L.parts : 0);
  L.row_scale = take(gradient ? piece * 4 : 0);
  // shares of the second product's tiles: no more than its tiles can be split into
  const size_t tiles = piece / kHeadTile * ((size_t)(s.d_model + kHeadTile - 1) / kHeadTile);
  const size_t items = tiles * kHeadMaxShares;
  L.part_items = gradient ? (int)(items < kHeadMaxItems ? items : kHeadMaxItems) : 0;
  L.part = take(few_tokens(s) ? (gradient ? (size_t)head_few_shares(s.d_model, s.vocab) * tokens * s.d_model * 4 : 0)
                             : (size_t)L.part_items * kHeadTile * kHeadTile * 4);
  L.total = off;
  return L;
}

struct HeadCall {
  const void *x, *w;
  const int32_t *labels, *t_index;
  const float *t_logit, *t_lse, *weights, *normalizer;
  float *loss, *lse, *totals;
  void* d_x;
};

mixlora_status_t run_head(const mixlora_head_shape_t* s, const HeadCall& c, void* workspace, size_t workspace_bytes,
                          void* stream) {
  if (!aligned(c.x, 16) || !aligned(c.w, 16) || !aligned_or_null(c.d_x, 16) || !aligned(c.loss, 4) ||
      !aligned_or_null(c.lse, 4) || !aligned_or_null(c.totals, 4) || !aligned_or_null(c.weights, 4) ||
      !aligned_or_null(c.normalizer, 4) || c.d_x == c.x)
    return MIXLORA_ERR_INVALID_ARG;
  const bool gradient = c.d_x != nullptr;
  const HeadLayout L = head_layout(*s, gradient);
  if (!aligned(workspace, 256) || workspace_bytes < L.total) return MIXLORA_ERR_WORKSPACE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  char* ws = reinterpret_cast<char*>(workspace);
  if (s->tokens == 0) {
    MIXLORA_TRY(cudaMemsetAsync(ws + L.state, 0, sizeof(HeadState), st));
    if (c.totals) MIXLORA_TRY(cudaMemsetAsync(c.totals, 0, 8, st));
    return MIXLORA_OK;
  }
  HeadArgs a;
  memset(&a, 0, sizeof(a));
  a.x = c.x; a.w = c.w; a.d_x = c.d_x;
  a.x_stride = stride_of(s->x_stride, s->d_model);
  a.w_stride = stride_of(s->w_stride, s->d_model);
  a.dx_stride = stride_of(s->d_x_stride, s->d_model);
  a.tokens = s->tokens; a.d = s->d_model; a.vocab = s->vocab; a.top = s->teacher_top ? s->teacher_top : 1;
  a.labels = c.labels; a.t_index = c.t_index; a.t_logit = c.t_logit; a.t_lse = c.t_lse;
  a.weights = c.weights; a.normalizer = c.normalizer;
  a.loss = c.loss; a.lse = c.lse; a.totals = c.totals;
  a.scale = s->scale; a.softcap = s->softcap; a.temperature = s->temperature; a.z_loss = s->z_loss;
  const bool cap = s->softcap > 0.f;
  a.logit_factor = cap ? s->scale / s->softcap : s->scale / s->temperature;
  a.cap_out = cap ? s->softcap / s->temperature : 0.f;
  a.to2 = (float)(1.44269504088896340736 * (cap ? (double)s->softcap : (double)s->scale) / (double)s->temperature);
  a.z_per_xw = (double)s->scale / (double)s->temperature;
  a.z_to_cap = cap ? (double)s->temperature / (double)s->softcap : 0.0;
  a.state = reinterpret_cast<HeadState*>(ws + L.state);
  a.row_token = reinterpret_cast<int32_t*>(ws + L.row_token);
  a.token_row = reinterpret_cast<int32_t*>(ws + L.token_row);
  a.list_out = reinterpret_cast<int32_t*>(ws + L.list);
  a.list = c.labels ? c.labels : a.list_out;
  a.list_q = reinterpret_cast<double*>(ws + L.list_q);
  a.rest_q = reinterpret_cast<double*>(ws + L.rest_q);
  a.list_n = reinterpret_cast<int32_t*>(ws + L.list_n);
  a.loss_part = reinterpret_cast<double*>(ws + L.loss_part);
  a.x_rows = ws + L.x_rows;
  a.w_parts = reinterpret_cast<bf16*>(ws + L.w_parts);
  a.z_listed = reinterpret_cast<float*>(ws + L.z_listed);
  a.stats = reinterpret_cast<float2*>(ws + L.stats);
  a.e = ws + L.e;
  a.e_part = (long long)L.piece * L.pitch;
  a.parts = L.parts;
  a.row_scale = reinterpret_cast<float*>(ws + L.row_scale);
  a.part = reinterpret_cast<float*>(ws + L.part);
  a.piece = L.piece; a.pitch = L.pitch; a.cols = L.cols; a.col_tiles = L.col_tiles;
  a.part_items = L.part_items;

  if (!c.labels) MIXLORA_TRY(launch_head_lists(a, st));
  // With no more tokens than a tile has rows, leaving some out saves nothing: rows are tokens, and nothing has to be numbered
  // (100 tokens of 32000 columns: 68 -> 64 us).
  a.few = s->tokens <= kHeadTile;
  const bool lists = !c.labels;
  if (few_tokens(*s)) {
    MIXLORA_TRY(launch_head_logits_few(a, !lists, st));
    MIXLORA_TRY(launch_head_join(a, st));
    if (gradient) MIXLORA_TRY(launch_head_grad_few(a, st));
    return MIXLORA_OK;
  }
  if (!a.few) MIXLORA_TRY(launch_head_scan(a, !lists, st));
  if (L.parts == 3) MIXLORA_TRY(launch_head_parts(a, a.few && !lists, st));
  for (int i = 0; i < L.pieces; ++i) {
    a.piece0 = i * L.piece;
    if (!a.few) MIXLORA_TRY(launch_head_gather(a, st));
    MIXLORA_TRY(launch_head_logits_tc(a, st));
    MIXLORA_TRY(launch_head_join(a, st));
    if (gradient) MIXLORA_TRY(launch_head_grad_tc(a, st));
  }
  return MIXLORA_OK;
}

}  // namespace
}  // namespace mixlora

using namespace mixlora;

extern "C" {

size_t mixlora_head_workspace_bytes(const mixlora_head_shape_t* shape, int with_gradient) {
  return check_head(shape) == MIXLORA_OK ? head_layout(*shape, with_gradient != 0).total : 0;
}

mixlora_status_t mixlora_head_loss(const mixlora_head_shape_t* shape, const void* x, const void* w, const int32_t* labels,
                                   const float* weights, const float* normalizer, float* loss, float* lse, float* totals,
                                   void* d_x, void* workspace, size_t workspace_bytes, void* stream) {
  const mixlora_status_t st = check_head(shape);
  if (st != MIXLORA_OK) return st;
  if (shape->teacher_top != 0 || !aligned(labels, 4)) return MIXLORA_ERR_INVALID_ARG;
  const HeadCall c{x, w, labels, nullptr, nullptr, nullptr, weights, normalizer, loss, lse, totals, d_x};
  return run_head(shape, c, workspace, workspace_bytes, stream);
}

mixlora_status_t mixlora_head_distill(const mixlora_head_shape_t* shape, const void* x, const void* w,
                                      const int32_t* teacher_index, const float* teacher_logit, const float* teacher_lse,
                                      const float* weights, const float* normalizer, float* loss, float* lse,
                                      float* totals, void* d_x, void* workspace, size_t workspace_bytes, void* stream) {
  const mixlora_status_t st = check_head(shape);
  if (st != MIXLORA_OK) return st;
  if (shape->teacher_top == 0 || !aligned(teacher_index, 4) || !aligned(teacher_logit, 4) || !aligned_or_null(teacher_lse, 4))
    return MIXLORA_ERR_INVALID_ARG;
  const HeadCall c{x, w, nullptr, teacher_index, teacher_logit, teacher_lse, weights, normalizer, loss, lse, totals, d_x};
  return run_head(shape, c, workspace, workspace_bytes, stream);
}

}  // extern "C"
