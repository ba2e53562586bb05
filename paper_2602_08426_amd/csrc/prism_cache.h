// What the serving entry points share (rotary positions, the paged cache, attention over it): argument checks, the
// descriptors as the kernels take them, where a row of a packed batch stands.
#pragma once

#include "prism_common.h"

namespace prism {

constexpr int kMaxPairs = kMaxHeadDim / 2;
// Limits of a call.  A grid's first dimension has fewer than 2^32 threads: 16 units of a token's head, 256 threads for each page of
// up to n / 32 + 2 s, for each row tile of up to rows / 128 + pairs.  Units of 256 sequences are added in 32 bits.
constexpr int kMaxTokens = 1 << 27;
constexpr int kMaxSeqs = 1 << 21;
constexpr int kMaxPlaces = 1 << 29;             // of a sequence
constexpr int kMaxRows = 1 << 30;               // tokens times q-heads (attention)
constexpr int kMaxSeqHeads = 1 << 22;           // pairs of a sequence and a kv head (attention)
constexpr int kMaxHeads = 1 << 14;              // Q, K and V heads together are a grid's second dimension
constexpr float kE4m3Max = 448.f;
constexpr int kMinScaleExponent = -120;         // of a page and head that holds zeros only

// ---- tensors [heads, tokens, d] with strides ---------------------------------------------------
struct Rows {
  uint16_t* p;
  int64_t head;            // elements
  int64_t token;
};
inline Rows rows_of(const prism_rows* r) {
  return r != nullptr ? Rows{static_cast<uint16_t*>(r->data), r->head_stride, r->token_stride} : Rows{nullptr, 0, 0};
}
inline int check_rows(const prism_rows* r, int heads, int tokens, int d, bool written) {
  if (r == nullptr || r->data == nullptr || ((uintptr_t)r->data & 15) != 0) return PRISM_ERR_INVALID_ARG;
  const bool by_head = heads > 1, by_token = tokens > 1;
  if (by_head && (r->head_stride < 0 || r->head_stride % 8 != 0)) return PRISM_ERR_INVALID_ARG;
  if (by_token && (r->token_stride < 0 || r->token_stride % 8 != 0)) return PRISM_ERR_INVALID_ARG;
  // so that no offset leaves 63 bits
  if ((by_head && r->head_stride > ((int64_t)1 << 62) / heads / 4) || (by_token && r->token_stride > ((int64_t)1 << 62) / tokens / 4))
    return PRISM_ERR_INVALID_ARG;
  if (!written) return PRISM_OK;
  const int64_t h = by_head ? r->head_stride : 0, t = by_token ? r->token_stride : 0;
  if ((by_head && h < d) || (by_token && t < d)) return PRISM_ERR_INVALID_ARG;
  if (by_head && by_token && h < (tokens - 1) * t + d && t < (heads - 1) * h + d) return PRISM_ERR_INVALID_ARG;
  return PRISM_OK;
}
// an output that starts where its input does has to be the input
inline int check_in_place(const prism_rows* in, const prism_rows* out, int heads, int tokens) {
  if (in->data != out->data) return PRISM_OK;
  if ((heads > 1 && in->head_stride != out->head_stride) || (tokens > 1 && in->token_stride != out->token_stride))
    return PRISM_ERR_INVALID_ARG;
  return PRISM_OK;
}
inline bool known_head_dim(int d) { return d == 64 || d == 128 || d == 256; }

// ---- rotary positions --------------------------------------------------------------------------
// theta'_j in turns per position: formed once on the host, in double.
struct RotaryTable {
  double turns[kMaxPairs];
  double offset;           // added to every position
  float magnitude;
  float sign;              // -1: the transposed map
  int rot;                 // dims that turn; 0 = none
  int half;                // pairs (j, j + rot/2)
};
inline int check_rotary(const prism_rotary* r, int head_dim) {
  if (r == nullptr) return PRISM_ERR_INVALID_ARG;
  if (r->rot_dim < 16 || r->rot_dim > head_dim || r->rot_dim % 16 != 0) return PRISM_ERR_INVALID_ARG;
  if (r->layout != PRISM_ROPE_INTERLEAVED && r->layout != PRISM_ROPE_HALF) return PRISM_ERR_INVALID_ARG;
  if (!(r->magnitude > 0.f) || !(r->magnitude < INFINITY)) return PRISM_ERR_INVALID_ARG;
  const prism_rope& f = r->freq;
  if (!(f.base > 1.0) || !(f.base < (double)INFINITY) || f.position_offset < 0 || f.position_offset >= 1 << 30) return PRISM_ERR_INVALID_ARG;
  if (f.yarn_native_len != 0 && (f.yarn_native_len < 0 || !(f.yarn_scale >= 1.0) || !(f.yarn_scale < (double)INFINITY) ||
                                 !(f.yarn_alpha >= 0.0) || !(f.yarn_beta > f.yarn_alpha)))
    return PRISM_ERR_INVALID_ARG;
  return PRISM_OK;
}
RotaryTable rotary_table(const prism_rotary* r, bool backward);    // r = NULL: nothing turns

// ---- the cache and its batch -------------------------------------------------------------------
struct CacheView {
  char* k;
  char* v;
  float* k_scale;
  float* v_scale;
  int64_t page_stride;     // bytes
  int32_t n_pages, h_kv, page, page_shift;
};
struct BatchView {
  const int32_t* cu;       // NULL: `each` new tokens for every sequence
  const int32_t* lengths;
  const int32_t* table;
  int32_t n_seqs, n_tokens, each, max_pages;
};
inline int check_cache(const prism_cache* c) {
  if (c == nullptr) return PRISM_ERR_INVALID_ARG;
  if (!known_head_dim(c->head_dim) || (c->page != 32 && c->page != 64 && c->page != 128)) return PRISM_ERR_UNSUPPORTED;
  if (c->dtype != PRISM_CACHE_BF16 && c->dtype != PRISM_CACHE_E4M3) return PRISM_ERR_UNSUPPORTED;
  if (c->n_pages <= 0 || c->n_kv_heads <= 0) return PRISM_ERR_INVALID_ARG;
  if (c->n_kv_heads > kMaxHeads) return PRISM_ERR_UNSUPPORTED;
  const int64_t least = (int64_t)c->n_kv_heads * c->page * c->head_dim;
  if (c->page_stride != 0 && (c->page_stride < least || c->page_stride % 16 != 0 || c->page_stride > ((int64_t)1 << 60) / c->n_pages))
    return PRISM_ERR_INVALID_ARG;
  return PRISM_OK;
}
inline int check_cache_memory(const prism_cache* c) {
  if (c->k == nullptr || c->v == nullptr || (((uintptr_t)c->k | (uintptr_t)c->v) & 15) != 0) return PRISM_ERR_INVALID_ARG;
  const bool scales = c->k_scale != nullptr && c->v_scale != nullptr;
  const bool none = c->k_scale == nullptr && c->v_scale == nullptr;
  return (c->dtype == PRISM_CACHE_E4M3 ? scales : none) ? PRISM_OK : PRISM_ERR_INVALID_ARG;
}
inline int check_batch(const prism_cache* c, const prism_batch* b) {
  if (b == nullptr) return PRISM_ERR_INVALID_ARG;
  if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_tokens <= 0 || b->max_pages <= 0) return PRISM_ERR_INVALID_ARG;
  if ((int64_t)b->max_pages * c->page > kMaxPlaces) return PRISM_ERR_UNSUPPORTED;
  if (b->n_tokens > kMaxTokens || b->n_seqs > kMaxSeqs) return PRISM_ERR_UNSUPPORTED;
  if (b->n_tokens == 0) return PRISM_OK;
  if (b->n_seqs == 0 || b->lengths == nullptr || b->page_table == nullptr) return PRISM_ERR_INVALID_ARG;
  if (b->cu_tokens == nullptr && (int64_t)b->n_seqs * b->max_tokens != b->n_tokens) return PRISM_ERR_INVALID_ARG;
  return PRISM_OK;
}
inline CacheView cache_view(const prism_cache* c) {
  const int64_t stride = c->page_stride != 0 ? c->page_stride : (int64_t)c->n_kv_heads * c->page * c->head_dim;
  CacheView v = {static_cast<char*>(c->k), static_cast<char*>(c->v), c->k_scale, c->v_scale,
                 stride * (c->dtype == PRISM_CACHE_E4M3 ? 1 : 2), c->n_pages, c->n_kv_heads, c->page, 0};
  while ((1 << v.page_shift) < c->page) ++v.page_shift;
  return v;
}
inline BatchView batch_view(const prism_batch* b) {
  return BatchView{b->cu_tokens, b->lengths, b->page_table, b->n_seqs, b->n_tokens, b->max_tokens, b->max_pages};
}

// ---- device ------------------------------------------------------------------------------------
// The rows of a sequence: whatever the offsets hold, 0 <= row0 <= row0 + n <= n_tokens.
struct SeqRows {
  int row0, n, length;     // length: tokens of the sequence, at least 0
};
__device__ __forceinline__ int row_start(const BatchView& b, int s) {
  return b.cu != nullptr ? min(max(b.cu[s], 0), b.n_tokens) : s * b.each;
}
__device__ __forceinline__ SeqRows seq_rows(const BatchView& b, int s) {
  SeqRows r;
  r.row0 = row_start(b, s);
  r.n = max(row_start(b, s + 1) - r.row0, 0);
  r.length = min(max(b.lengths[s], 0), 0x3fffffff);
  return r;
}
// The last sequence s with mul * (start of s) / div + extra * s <= at (sequence 0 if there is none): a binary search.
__device__ __forceinline__ int seq_at(const BatchView& b, int at, int mul, int div_shift, int extra) {
  int lo = 0, hi = b.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    const int64_t start = (((int64_t)row_start(b, mid) * mul) >> div_shift) + (int64_t)extra * mid;
    if (start <= at) lo = mid; else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const f32x2 x = {a, b};
  const bf16x2 y = __builtin_convertvector(x, bf16x2);
  return __builtin_bit_cast(uint32_t, y);
}

}  // namespace prism
