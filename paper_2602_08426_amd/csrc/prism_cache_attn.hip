// Attention of new tokens over the paged cache (gfx950): prism_cache_attn.
#include "prism_cache.h"

namespace prism {

// One workgroup for a new token and a q-head: 256 keys at a time, one a thread, then their values by dims.
template <int D, bool kE4m3>
__global__ __launch_bounds__(256) void cache_attn_simple_kernel(Rows q, Rows out, float* __restrict__ lse, CacheView cache,
                                                                BatchView batch, int h, int window, int sinks, float scale) {
  __shared__ float s_q[D], s_p[256], s_red[8];
  __shared__ int s_id[256];
  const int64_t token = blockIdx.x;
  const int hq = blockIdx.y, kv = hq / (h / cache.h_kv), t = threadIdx.x;
  const int s = seq_at(batch, (int)token, 1, 0, 0);
  const SeqRows r = seq_rows(batch, s);
  const int i = (int)token - r.row0;
  if (i < 0 || i >= r.n || i >= batch.each) return;
  const int pos = r.length - r.n + i;
  for (int d = t; d < D; d += 256) s_q[d] = bf16_bits_to_float(q.p[hq * q.head + token * q.token + d]);
  __syncthreads();
  const int end = min(pos + 1, batch.max_pages << cache.page_shift);
  const int low = window > 0 ? max(pos - window + 1, 0) : 0;
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int j0 = 0; j0 < end; j0 += 256) {
    if (j0 >= sinks && j0 + 256 <= low) continue;
    const int j = j0 + t;
    int id = -1;
    if (j < end && (j >= low || j < sinks)) id = batch.table[(int64_t)s * batch.max_pages + (j >> cache.page_shift)];
    const bool sees = id >= 0 && id < cache.n_pages;
    float x = -INFINITY;
    if (sees) {
      const char* row = cache.k + id * cache.page_stride + ((int64_t)kv * cache.page + (j & (cache.page - 1))) * (D * (kE4m3 ? 1 : 2));
      x = 0.f;
      for (int d = 0; d < D; d += 4) {
        if (kE4m3) {
          const int w = *reinterpret_cast<const int*>(row + d);
          const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
          x += s_q[d] * a[0] + s_q[d + 1] * a[1] + s_q[d + 2] * b[0] + s_q[d + 3] * b[1];
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(row + 2 * d);
          x += s_q[d] * __uint_as_float(w.x << 16) + s_q[d + 1] * __uint_as_float(w.x & 0xFFFF0000u) +
               s_q[d + 2] * __uint_as_float(w.y << 16) + s_q[d + 3] * __uint_as_float(w.y & 0xFFFF0000u);
        }
      }
      if (kE4m3) x *= cache.k_scale[(int64_t)id * cache.h_kv + kv];
      x *= scale;
    }
    float top = wave_max(x);
    if ((t & 63) == 0) s_red[t >> 6] = top;
    __syncthreads();
    top = fmaxf(m, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
    const float base = top == -INFINITY ? 0.f : top;
    const float p = sees ? expf(x - base) : 0.f;
    const float sum = wave_sum(p);
    if ((t & 63) == 0) s_red[4 + (t >> 6)] = sum;
    s_p[t] = p;
    s_id[t] = sees ? id : -1;
    __syncthreads();
    const float keep = expf(m - base);
    l = l * keep + (s_red[4] + s_red[5] + s_red[6] + s_red[7]);
    m = top;
    if (t < D) {
      o *= keep;
      for (int i2 = 0; i2 < 256; ++i2) {
        const int key = s_id[i2];
        if (key < 0) continue;
        const int64_t at = key * cache.page_stride + ((int64_t)kv * cache.page + ((j0 + i2) & (cache.page - 1))) * (D * (kE4m3 ? 1 : 2));
        float v;
        if (kE4m3)
          v = __builtin_amdgcn_cvt_pk_f32_fp8((int)*reinterpret_cast<const uint8_t*>(cache.v + at + t), false)[0] *
              cache.v_scale[(int64_t)key * cache.h_kv + kv];
        else
          v = bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(cache.v + at + 2 * t));
        o += s_p[i2] * v;
      }
    }
    __syncthreads();
  }
  if (t < D) {
    const __bf16 y = (__bf16)(l == 0.f ? 0.f : o / l);
    out.p[hq * out.head + token * out.token + t] = __builtin_bit_cast(uint16_t, y);
  }
  if (t == 0 && lse != nullptr) lse[(int64_t)hq * batch.n_tokens + token] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace prism

using namespace prism;

static int check_attn(const prism_cache* cache, const prism_batch* batch, int n_q_heads) {
  int rc = check_cache(cache);
  if (rc != PRISM_OK || (rc = check_batch(cache, batch)) != PRISM_OK) return rc;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0) return PRISM_ERR_INVALID_ARG;
  return PRISM_OK;
}

extern "C" int prism_cache_attn_workspace_bytes(const prism_cache* cache, const prism_batch* batch, int n_q_heads, size_t* bytes) {
  const int rc = check_attn(cache, batch, n_q_heads);
  if (rc != PRISM_OK) return rc;
  if (bytes == nullptr) return PRISM_ERR_INVALID_ARG;
  *bytes = 256;
  return PRISM_OK;
}

template <int D>
static void launch_simple(const prism_cache* c, const prism_batch* b, const prism_cache_attn_params* p, const prism_rows* q, const prism_rows* out,
                          float* lse, float scale, hipStream_t st) {
  const dim3 grid(b->n_tokens, p->n_q_heads);
  if (c->dtype == PRISM_CACHE_E4M3)
    hipLaunchKernelGGL((cache_attn_simple_kernel<D, true>), grid, dim3(256), 0, st, rows_of(q), rows_of(out), lse, cache_view(c),
                       batch_view(b), p->n_q_heads, p->window, p->sinks, scale);
  else
    hipLaunchKernelGGL((cache_attn_simple_kernel<D, false>), grid, dim3(256), 0, st, rows_of(q), rows_of(out), lse, cache_view(c),
                       batch_view(b), p->n_q_heads, p->window, p->sinks, scale);
}

extern "C" int prism_cache_attn(const prism_cache* cache, const prism_batch* batch, const prism_cache_attn_params* params,
                                const prism_rows* q, const prism_rows* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (params == nullptr) return PRISM_ERR_INVALID_ARG;
  int rc = check_attn(cache, batch, params->n_q_heads);
  if (rc != PRISM_OK) return rc;
  if (params->window < 0 || params->sinks < 0 || !(params->scale >= 0.f) || !(params->scale < INFINITY)) return PRISM_ERR_INVALID_ARG;
  const int d = cache->head_dim;
  if (batch->n_tokens == 0) return PRISM_OK;
  if ((rc = check_cache_memory(cache)) != PRISM_OK || (rc = check_rows(q, params->n_q_heads, batch->n_tokens, d, false)) != PRISM_OK ||
      (rc = check_rows(out, params->n_q_heads, batch->n_tokens, d, true)) != PRISM_OK ||
      (rc = check_in_place(q, out, params->n_q_heads, batch->n_tokens)) != PRISM_OK)
    return rc;
  size_t need = 0;
  rc = prism_cache_attn_workspace_bytes(cache, batch, params->n_q_heads, &need);
  if (rc != PRISM_OK) return rc;
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need) return PRISM_ERR_WORKSPACE;
  const float scale = params->scale > 0.f ? params->scale : 1.f / sqrtf((float)d);
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (d) {
    case 64: launch_simple<64>(cache, batch, params, q, out, lse, scale, st); break;
    case 128: launch_simple<128>(cache, batch, params, q, out, lse, scale, st); break;
    default: launch_simple<256>(cache, batch, params, q, out, lse, scale, st); break;
  }
  return launch_status();
}
