// C ABI of the rotary positions and the masked attention: argument checks, workspace layout, launches.
#include <math.h>
#include <string.h>

#include "attention.cuh"
#include "rope.cuh"

namespace mixlora {
namespace {

bool aligned(const void* p, size_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool dtype_ok(int32_t d) { return d == MIXLORA_DTYPE_BF16 || d == MIXLORA_DTYPE_FP32; }

#define MIXLORA_TRY(expr)                               \
  do {                                                  \
    if ((expr) != cudaSuccess) return MIXLORA_ERR_CUDA; \
  } while (0)

// A stride as given or, for 0, dense; -1 if rows would overlap
long long stride_of(int64_t given, int heads, int dim) {
  const long long dense = (long long)heads * dim;
  if (given == 0) return dense;
  return given >= dense ? (long long)given : -1;
}

// ---- rotary positions ----
mixlora_status_t rope(const mixlora_rope_shape_t* s, const void* q, const void* k, const int32_t* positions,
                      const double* inv_freq, void* q_out, void* k_out, int backward, void* stream) {
  if (!s || s->struct_size != sizeof(mixlora_rope_shape_t) || s->reserved != 0) return MIXLORA_ERR_INVALID_ARG;
  if (s->tokens < 0 || s->q_heads <= 0 || s->k_heads < 0 || s->head_dim <= 0 || !dtype_ok(s->dtype) ||
      (s->layout != MIXLORA_ROPE_HALF && s->layout != MIXLORA_ROPE_INTERLEAVED) || !isfinite(s->amplitude) ||
      s->rotary_dim < 2 || s->rotary_dim > s->head_dim || s->rotary_dim % 2)
    return MIXLORA_ERR_INVALID_ARG;
  if (s->head_dim % 8 || s->head_dim > 512 || s->q_heads > 65536 || s->k_heads > 65536) return MIXLORA_ERR_UNSUPPORTED;
  const long long strides[] = {stride_of(s->q_stride, s->q_heads, s->head_dim), stride_of(s->k_stride, s->k_heads, s->head_dim),
                               stride_of(s->q_out_stride, s->q_heads, s->head_dim),
                               stride_of(s->k_out_stride, s->k_heads, s->head_dim)};
  for (long long v : strides) {
    if (v < 0) return MIXLORA_ERR_INVALID_ARG;
    if (v % 8) return MIXLORA_ERR_UNSUPPORTED;
  }
  if (!aligned(q, 16) || !aligned(q_out, 16) || !aligned(inv_freq, 8)) return MIXLORA_ERR_INVALID_ARG;
  if (s->k_heads && (!aligned(k, 16) || !aligned(k_out, 16))) return MIXLORA_ERR_INVALID_ARG;
  if (positions && !aligned(positions, 4)) return MIXLORA_ERR_INVALID_ARG;
  if ((q == q_out && strides[0] != strides[2]) || (s->k_heads && k == k_out && strides[1] != strides[3]))
    return MIXLORA_ERR_INVALID_ARG;
  if (s->tokens == 0) return MIXLORA_OK;
  RopeArgs p;
  memset(&p, 0, sizeof(p));
  p.q = q; p.k = k; p.q_out = q_out; p.k_out = k_out;
  p.q_stride = strides[0]; p.k_stride = strides[1]; p.q_out_stride = strides[2]; p.k_out_stride = strides[3];
  p.positions = positions; p.inv_freq = inv_freq; p.amplitude = s->amplitude;
  p.tokens = s->tokens; p.q_heads = s->q_heads; p.k_heads = s->k_heads; p.head_dim = s->head_dim;
  p.pairs = s->rotary_dim / 2;
  const bool in_place = q == q_out && (s->k_heads == 0 || k == k_out);
  p.copied = in_place ? 0 : s->head_dim - s->rotary_dim;
  p.backward = backward;
  MIXLORA_TRY(launch_rope(p, s->dtype == MIXLORA_DTYPE_BF16, s->layout == MIXLORA_ROPE_INTERLEAVED,
                          reinterpret_cast<cudaStream_t>(stream)));
  return MIXLORA_OK;
}

// ---- attention ----
mixlora_status_t check_attention(const mixlora_attention_shape_t* s) {
  if (!s || s->struct_size != sizeof(mixlora_attention_shape_t)) return MIXLORA_ERR_INVALID_ARG;
  if (s->n_seqs < 0 || s->q_rows < 0 || s->k_rows < 0 || s->max_q_len < 0 || s->max_k_len < 0 || s->q_heads <= 0 ||
      s->kv_heads <= 0 || s->head_dim <= 0 || s->window < 0 || (s->causal != 0 && s->causal != 1) || !dtype_ok(s->dtype))
    return MIXLORA_ERR_INVALID_ARG;
  if (s->q_heads % s->kv_heads) return MIXLORA_ERR_INVALID_ARG;
  if (!isfinite(s->scale) || s->scale <= 0.f || !isfinite(s->softcap) || s->softcap < 0.f) return MIXLORA_ERR_INVALID_ARG;
  // the factors that the kernels form of them, in fp32: none may overflow, and a cap's may not lose bits below the normal
  // range, since a large number multiplies what is left
  if (!isfinite(s->scale * kLog2e)) return MIXLORA_ERR_INVALID_ARG;
  if (s->softcap > 0.f && (!isnormal(s->scale / s->softcap) || !isnormal(s->softcap * kLog2e))) return MIXLORA_ERR_INVALID_ARG;
  const long long strides[] = {stride_of(s->q_stride, s->q_heads, s->head_dim), stride_of(s->k_stride, s->kv_heads, s->head_dim),
                               stride_of(s->v_stride, s->kv_heads, s->head_dim), stride_of(s->o_stride, s->q_heads, s->head_dim)};
  for (long long v : strides)
    if (v < 0) return MIXLORA_ERR_INVALID_ARG;
  if (s->head_dim % 8 || s->head_dim > MIXLORA_MAX_HEAD_DIM) return MIXLORA_ERR_UNSUPPORTED;
  for (long long v : strides)
    if (v % 8 || v > (1LL << 36)) return MIXLORA_ERR_UNSUPPORTED;
  if (s->q_rows > (1 << 30) || s->k_rows > (1 << 30) || s->n_seqs > (1 << 24) || s->q_heads > 65536)
    return MIXLORA_ERR_UNSUPPORTED;
  return MIXLORA_OK;
}

// Rows of a sequence that share a key head, if the form for few rows takes them, else 0
int few_rows(const mixlora_attention_shape_t& s) {
  const long long rows = (long long)s.max_q_len * (s.q_heads / s.kv_heads);
  return rows > 0 && rows <= kFewRowsMax ? (int)rows : 0;
}
FewSplits splits_of(const mixlora_attention_shape_t& s) {
  return attn_few_splits(s.n_seqs, s.kv_heads, few_rows(s), s.k_rows, s.max_k_len);
}

// Tiles of `tile` rows that `rows` rows in n_seqs sequences can have at most
int tile_capacity(int rows, int n_seqs, int tile) { return (rows + tile - 1) / tile + n_seqs; }

struct AttnLayout { size_t status, part, lse2, delta, q_tiles, k_tiles, q_first, k_first, total; };
AttnLayout attention_layout(const mixlora_attention_shape_t& s, bool backward) {
  AttnLayout L;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
  L.status = take(256);
  const int rows = few_rows(s);
  const FewSplits sp = rows ? splits_of(s) : FewSplits{1, false};
  const size_t chunks = (size_t)(rows + kFewRows - 1) / kFewRows;
  L.part = take(sp.count > 1 && !sp.cluster ? (size_t)s.n_seqs * s.kv_heads * chunks * sp.count * kFewRows * (s.head_dim + 3) * 4 : 0);
  const size_t per_row = backward ? (size_t)s.q_heads * s.q_rows * 4 : 0;
  L.lse2 = take(per_row);
  L.delta = take(per_row);
  // plans of the tensor-core kernels; their tile counts sit in the status block
  const bool tiled = s.dtype == MIXLORA_DTYPE_BF16 && (backward || !rows);
  const size_t seqs = tiled ? (size_t)s.n_seqs : 0;
  L.q_tiles = take(tiled ? (size_t)tile_capacity(s.q_rows, s.n_seqs, backward ? kBwdTile : kFwdTile) * sizeof(AttnTile) : 0);
  L.k_tiles = take(tiled && backward ? (size_t)tile_capacity(s.k_rows, s.n_seqs, kBwdTile) * sizeof(AttnTile) : 0);
  L.q_first = take(seqs * 4);
  L.k_first = take(backward ? seqs * 4 : 0);
  L.total = off;
  return L;
}

// Fills in the plans' places; returns the number of jobs
int plan_jobs(const mixlora_attention_shape_t& s, const AttnLayout& L, char* ws, bool backward, AttnArgs* a,
              AttnPlanJob* jobs) {
  int32_t* counts = reinterpret_cast<int32_t*>(ws + L.status) + 8;
  jobs[0] = AttnPlanJob{reinterpret_cast<AttnTile*>(ws + L.q_tiles), counts, reinterpret_cast<int32_t*>(ws + L.q_first),
                        backward ? kBwdTile : kFwdTile, tile_capacity(s.q_rows, s.n_seqs, backward ? kBwdTile : kFwdTile), 0};
  jobs[1] = AttnPlanJob{reinterpret_cast<AttnTile*>(ws + L.k_tiles), counts + 1, reinterpret_cast<int32_t*>(ws + L.k_first),
                        kBwdTile, tile_capacity(s.k_rows, s.n_seqs, kBwdTile), 1};
  a->q_tiles = jobs[0].table; a->n_q_tiles = jobs[0].count;
  a->k_tiles = jobs[1].table; a->n_k_tiles = jobs[1].count;
  return backward ? 2 : 1;
}

mixlora_status_t attention_args(const mixlora_attention_shape_t* s, const mixlora_attention_mask_t* m, const void* q,
                                const void* k, const void* v, const void* o, const void* ws, size_t ws_bytes,
                                bool backward, AttnArgs* a) {
  mixlora_status_t st = check_attention(s);
  if (st != MIXLORA_OK) return st;
  if (!m || !aligned(m->q_off, 4) || !aligned(m->k_off, 4)) return MIXLORA_ERR_INVALID_ARG;
  const void* opt[] = {m->k_len, m->prefix, m->slopes};
  for (const void* x : opt)
    if (x && !aligned(x, 4)) return MIXLORA_ERR_INVALID_ARG;
  const void* req[] = {q, k, v, o};
  for (const void* x : req)
    if (!aligned(x, 16)) return MIXLORA_ERR_INVALID_ARG;
  if (!aligned(ws, 256) || ws_bytes < attention_layout(*s, backward).total) return MIXLORA_ERR_WORKSPACE;
  memset(a, 0, sizeof(*a));
  a->q = q; a->k = k; a->v = v;
  a->q_off = m->q_off; a->k_off = m->k_off; a->k_len = m->k_len; a->prefix = m->prefix; a->slopes = m->slopes;
  a->q_stride = stride_of(s->q_stride, s->q_heads, s->head_dim);
  a->k_stride = stride_of(s->k_stride, s->kv_heads, s->head_dim);
  a->v_stride = stride_of(s->v_stride, s->kv_heads, s->head_dim);
  a->o_stride = stride_of(s->o_stride, s->q_heads, s->head_dim);
  a->n_seqs = s->n_seqs; a->q_rows = s->q_rows; a->k_rows = s->k_rows;
  a->q_heads = s->q_heads; a->kv_heads = s->kv_heads; a->group = s->q_heads / s->kv_heads; a->head_dim = s->head_dim;
  a->causal = s->causal; a->max_q_len = s->max_q_len;
  // a row is at most lk - 1 behind and lq - 1 before a key: a window that wide hides nothing, and with those below 2^30 no
  // position less a window leaves 32 bits
  a->window = s->window >= s->q_rows && s->window >= s->k_rows ? 0 : s->window;
  a->scale = s->scale; a->softcap = s->softcap;
  return MIXLORA_OK;
}

}  // namespace
}  // namespace mixlora

using namespace mixlora;

extern "C" {

mixlora_status_t mixlora_rope_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor,
                                          double low_turns, double high_turns, int32_t original_positions,
                                          double* inv_freq, void* stream) {
  if (rotary_dim < 2 || rotary_dim % 2 || !aligned(inv_freq, 8)) return MIXLORA_ERR_INVALID_ARG;
  if (!isfinite(theta) || theta <= 0.0 || !isfinite(factor) || factor <= 0.0) return MIXLORA_ERR_INVALID_ARG;
  if (scaling < MIXLORA_ROPE_SCALE_NONE || scaling > MIXLORA_ROPE_SCALE_PARTS) return MIXLORA_ERR_INVALID_ARG;
  if (scaling == MIXLORA_ROPE_SCALE_PARTS &&
      !(low_turns >= 0.0 && low_turns < high_turns && isfinite(high_turns) && original_positions > 0))
    return MIXLORA_ERR_INVALID_ARG;
  if (rotary_dim > 512) return MIXLORA_ERR_UNSUPPORTED;
  MIXLORA_TRY(launch_rope_frequencies(rotary_dim / 2, theta, scaling, factor, low_turns, high_turns,
                                      (double)original_positions, inv_freq, reinterpret_cast<cudaStream_t>(stream)));
  return MIXLORA_OK;
}

mixlora_status_t mixlora_rope_forward(const mixlora_rope_shape_t* shape, const void* q, const void* k,
                                      const int32_t* positions, const double* inv_freq, void* q_out, void* k_out,
                                      void* stream) {
  return rope(shape, q, k, positions, inv_freq, q_out, k_out, 0, stream);
}

mixlora_status_t mixlora_rope_backward(const mixlora_rope_shape_t* shape, const void* d_q_out, const void* d_k_out,
                                       const int32_t* positions, const double* inv_freq, void* d_q, void* d_k,
                                       void* stream) {
  return rope(shape, d_q_out, d_k_out, positions, inv_freq, d_q, d_k, 1, stream);
}

size_t mixlora_attention_workspace_bytes(const mixlora_attention_shape_t* shape, int for_backward) {
  return check_attention(shape) == MIXLORA_OK ? attention_layout(*shape, for_backward != 0).total : 0;
}

mixlora_status_t mixlora_attention_forward(const mixlora_attention_shape_t* shape, const mixlora_attention_mask_t* mask,
                                           const void* q, const void* k, const void* v, void* o, float* lse,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  AttnArgs a;
  mixlora_status_t st = attention_args(shape, mask, q, k, v, o, workspace, workspace_bytes, false, &a);
  if (st != MIXLORA_OK) return st;
  if (lse && !aligned(lse, 4)) return MIXLORA_ERR_INVALID_ARG;
  const AttnLayout L = attention_layout(*shape, false);
  cudaStream_t cs = reinterpret_cast<cudaStream_t>(stream);
  char* ws = reinterpret_cast<char*>(workspace);
  a.out = o;
  a.lse = lse;
  a.status = reinterpret_cast<int32_t*>(ws + L.status);
  const bool bf16_mode = shape->dtype == MIXLORA_DTYPE_BF16;
  if (few_rows(*shape) && a.n_seqs > 0 && a.q_rows > 0) {    // sets the status word itself
    MIXLORA_TRY(launch_attn_few(a, bf16_mode, splits_of(*shape), reinterpret_cast<float*>(ws + L.part), cs));
    return MIXLORA_OK;
  }
  if (!bf16_mode || a.n_seqs == 0 || a.q_rows == 0) {
    MIXLORA_TRY(cudaMemsetAsync(a.status, 0, 256, cs));
    if (a.n_seqs == 0 || a.q_rows == 0) return MIXLORA_OK;
    MIXLORA_TRY(launch_attn_forward_simt(a, cs));
    return MIXLORA_OK;
  }
  AttnPlanJob jobs[2];
  const int n_jobs = plan_jobs(*shape, L, ws, false, &a, jobs);
  MIXLORA_TRY(launch_attn_plan(a, jobs, n_jobs, cs));        // clears the status word
  MIXLORA_TRY(launch_attn_forward_tc(a, cs));
  return MIXLORA_OK;
}

mixlora_status_t mixlora_attention_backward(const mixlora_attention_shape_t* shape, const mixlora_attention_mask_t* mask,
                                            const void* q, const void* k, const void* v, const void* o,
                                            const float* lse, const void* d_o, void* workspace, size_t workspace_bytes,
                                            void* d_q, void* d_k, void* d_v, void* stream) {
  AttnArgs a;
  mixlora_status_t st = attention_args(shape, mask, q, k, v, o, workspace, workspace_bytes, true, &a);
  if (st != MIXLORA_OK) return st;
  const void* req[] = {d_o, d_q, d_k, d_v};
  for (const void* x : req)
    if (!aligned(x, 16)) return MIXLORA_ERR_INVALID_ARG;
  if (!aligned(lse, 4)) return MIXLORA_ERR_INVALID_ARG;
  const AttnLayout L = attention_layout(*shape, true);
  cudaStream_t cs = reinterpret_cast<cudaStream_t>(stream);
  char* ws = reinterpret_cast<char*>(workspace);
  float* lse2 = reinterpret_cast<float*>(ws + L.lse2);
  float* delta = reinterpret_cast<float*>(ws + L.delta);
  a.o = o; a.d_o = d_o; a.dq = d_q; a.dk = d_k; a.dv = d_v;
  a.lse = const_cast<float*>(lse);
  a.lse2 = lse2;
  a.delta = delta;
  a.status = reinterpret_cast<int32_t*>(ws + L.status);
  const bool bf16_mode = shape->dtype == MIXLORA_DTYPE_BF16;
  if (!bf16_mode || a.n_seqs == 0) {
    MIXLORA_TRY(cudaMemsetAsync(a.status, 0, 256, cs));
    if (a.n_seqs == 0) return MIXLORA_OK;
    MIXLORA_TRY(launch_attn_delta(a, bf16_mode, lse2, delta, cs));
    MIXLORA_TRY(launch_attn_backward_simt(a, cs));
    return MIXLORA_OK;
  }
  AttnPlanJob jobs[2];
  const int n_jobs = plan_jobs(*shape, L, ws, true, &a, jobs);
  MIXLORA_TRY(launch_attn_plan(a, jobs, n_jobs, cs));        // clears the status word
  MIXLORA_TRY(launch_attn_delta(a, bf16_mode, lse2, delta, cs));
  MIXLORA_TRY(launch_attn_backward_tc(a, cs));
  return MIXLORA_OK;
}

}  // extern "C"
