// Rotary positions and the paged cache of libprism (gfx950): prism_rotate, prism_cache_append.
//
// A unit is 16 dims of one token and head: 8 pairs and two 16-byte pieces (interleaved: dims 16u .. 16u+15; half: dims
// 8u .. 8u+7 and rot/2 + 8u ..).  A thread owns a unit of a token and goes through heads with it, so that the angles of its
// pairs are formed once for all of them.
//
// Both are bound by the bytes: each value is read once and written once, and the counters show nothing beyond that.  Measured
// (kernel alone; a large copy moves 5.0 TB/s): rotation of 32768 tokens of 28/4 heads, d = 128, 537 MB, 99 us = 5.4 TB/s; 20011 of 32/8
// heads inside a projection, half of the dims, 410 MB, 88 us = 4.7; 32768 of 8 kv heads to bf16 pages, 268 MB, 46 us (59 in a row of calls) = 4.6;
// 34794 of 8 kv heads to e4m3 pages and 32 q-heads, 784 MB, 65 + 109 us in the profiler, 160 in a row of calls = 4.9.  A call of one
// token is a kernel of 4 us.
#include "prism_cache.h"

#include <cmath>

namespace prism {

RotaryTable rotary_table(const prism_rotary* r, bool backward) {
  RotaryTable t = {};
  t.magnitude = t.sign = 1.f;
  if (r == nullptr) return t;
  const double two_pi = 6.283185307179586;
  t.rot = r->rot_dim;
  t.half = r->layout == PRISM_ROPE_HALF;
  t.magnitude = r->magnitude;
  t.sign = backward ? -1.f : 1.f;
  t.offset = r->freq.position_offset;
  for (int j = 0; j < t.rot / 2; ++j) {
    double theta = std::pow(r->freq.base, -2.0 * j / t.rot);
    if (r->freq.yarn_native_len != 0) {
      double gamma = (r->freq.yarn_native_len * theta / two_pi - r->freq.yarn_alpha) / (r->freq.yarn_beta - r->freq.yarn_alpha);
      gamma = gamma < 0.0 ? 0.0 : (gamma > 1.0 ? 1.0 : gamma);
      theta = (1.0 - gamma) * theta / r->freq.yarn_scale + gamma * theta;
    }
    t.turns[j] = theta / two_pi;
  }
  return t;
}

// cos and sin (times the magnitude) of the 8 pairs of unit u at a position.  The angle in turns is formed and reduced in
// fp64 (a position of 1e6 at 0.16 turns needs 2^-40 of it), the functions are evaluated in fp32.
struct Turn {
  float c[8], s[8];
};
__device__ __forceinline__ Turn turn_of(const RotaryTable& t, int u, double position) {
  Turn a;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const double x = (position + t.offset) * t.turns[8 * u + j];
    float c, s;
    sincospif(2.f * (float)(x - rint(x)), &s, &c);
    a.c[j] = c * t.magnitude;
    a.s[j] = s * t.magnitude * t.sign;
  }
  return a;
}

// A unit as 16 values: the first and second 8 dims of memory.
struct Unit {
  uint4 a, b;
};
// where the second piece of unit u lies, and the first
struct Places {
  int a, b;
  bool turns;
};
__device__ __forceinline__ Places places_of(const RotaryTable& t, int u) {
  const bool turns = u < t.rot / 16;
  if (turns && t.half) return Places{8 * u, t.rot / 2 + 8 * u, true};
  return Places{16 * u, 16 * u + 8, turns};
}
__device__ __forceinline__ Unit load_unit(const uint16_t* row, const Places& p) {
  return Unit{*reinterpret_cast<const uint4*>(row + p.a), *reinterpret_cast<const uint4*>(row + p.b)};
}
__device__ __forceinline__ void store_unit(uint16_t* row, const Places& p, const Unit& u) {
  *reinterpret_cast<uint4*>(row + p.a) = u.a;
  *reinterpret_cast<uint4*>(row + p.b) = u.b;
}
// the 16 values in fp32, turned; x[0..7] belong to the first piece
__device__ __forceinline__ void turned_values(const RotaryTable& t, const Unit& u, bool turns, const Turn& a, float x[16]) {
  const uint32_t w[8] = {u.a.x, u.a.y, u.a.z, u.a.w, u.b.x, u.b.y, u.b.z, u.b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
  if (!turns) return;
  if (t.half) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = x[j], q = x[8 + j];
      x[j] = p * a.c[j] - q * a.s[j];
      x[8 + j] = p * a.s[j] + q * a.c[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = x[2 * j], q = x[2 * j + 1];
      x[2 * j] = p * a.c[j] - q * a.s[j];
      x[2 * j + 1] = p * a.s[j] + q * a.c[j];
    }
  }
}
__device__ __forceinline__ Unit turned_unit(const RotaryTable& t, const Unit& u, bool turns, const Turn& a) {
  if (!turns) return u;                              // bits as they are
  float x[16];
  turned_values(t, u, turns, a, x);
  Unit y;
  y.a = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
  y.b = make_uint4(bf16_pair(x[8], x[9]), bf16_pair(x[10], x[11]), bf16_pair(x[12], x[13]), bf16_pair(x[14], x[15]));
  return y;
}

// ---- rows to rows, rows to bf16 pages ------------------------------------------------------------
struct RowJob {
  Rows q_in, q_out, k_in, k_out, v_in;
  int n_q, n_k, n_v;       // heads; with pages n_v = n_k, without them 0
  int n_tokens;
};
// kPaged: the tokens belong to the sequences of a batch and K and V go to their pages.
template <int D, bool kPaged>
__global__ __launch_bounds__(256) void rows_kernel(RowJob job, RotaryTable rot, const int32_t* __restrict__ positions,
                                                   CacheView cache, BatchView batch, int heads_each, int heads_first) {
  constexpr int U = D / 16;
  // heads_first: neighbouring workgroups have the same tokens and the next heads, otherwise the next tokens
  const int group = heads_first ? blockIdx.x : blockIdx.y;
  const int64_t idx = (int64_t)(heads_first ? blockIdx.y : blockIdx.x) * 256 + threadIdx.x;
  const int u = (int)(idx % U);
  const int64_t token = idx / U;
  if (token >= job.n_tokens) return;
  double position = (double)token;
  int64_t place = -1;                                // of the token in its page pool, bytes without the head; -1: none
  bool mine = true;                                  // the token belongs to a sequence
  if (kPaged) {
    const int s = seq_at(batch, (int)token, 1, 0, 0);
    const SeqRows r = seq_rows(batch, s);
    const int i = (int)token - r.row0;
    mine = i >= 0 && i < r.n;
    const int pos = r.length - r.n + i;
    position = pos;
    const int page = pos >> cache.page_shift;
    if (mine && pos >= 0 && page < batch.max_pages) {
      const int id = batch.table[(int64_t)s * batch.max_pages + page];
      if (id >= 0 && id < cache.n_pages) place = id * cache.page_stride + (int64_t)(pos & (cache.page - 1)) * (D * 2);
    }
  } else if (positions != nullptr) {
    position = positions[token];
  }
  if (!mine) return;
  const Places at = places_of(rot, u);
  const Places plain = Places{16 * u, 16 * u + 8, false};
  // Heads are taken kAtOnce at a time, all loads in front of the first store: the outputs may be the inputs, so that the
  // compiler keeps a load behind the store in front of it, and a thread waited for the memory at every head.
  constexpr int kAtOnce = 4;
  const int first = group * heads_each, last = min(first + heads_each, job.n_q + job.n_k + job.n_v);
  Turn turn = {};
  bool formed = false;
  for (int h0 = first; h0 < last; h0 += kAtOnce) {
    Unit x[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int hd = h0 + i;
      if (hd >= last) break;
      if (hd < job.n_q)
        x[i] = load_unit(job.q_in.p + hd * job.q_in.head + token * job.q_in.token, at);
      else if (hd < job.n_q + job.n_k)
        x[i] = load_unit(job.k_in.p + (hd - job.n_q) * job.k_in.head + token * job.k_in.token, at);
      else
        x[i] = load_unit(job.v_in.p + (hd - job.n_q - job.n_k) * job.v_in.head + token * job.v_in.token, plain);
    }
    if (!formed && at.turns) turn = turn_of(rot, u, position);      // while the first loads are under way
    formed = true;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int hd = h0 + i;
      if (hd >= last) break;
      if (hd < job.n_q) {
        store_unit(job.q_out.p + hd * job.q_out.head + token * job.q_out.token, at, turned_unit(rot, x[i], at.turns, turn));
      } else if (hd < job.n_q + job.n_k) {
        const int kv = hd - job.n_q;
        const Unit y = turned_unit(rot, x[i], at.turns, turn);
        if (!kPaged)
          store_unit(job.k_out.p + kv * job.k_out.head + token * job.k_out.token, at, y);
        else if (place >= 0)
          store_unit(reinterpret_cast<uint16_t*>(cache.k + place + (int64_t)kv * cache.page * (D * 2)), at, y);
      } else if (place >= 0) {
        const int kv = hd - job.n_q - job.n_k;
        store_unit(reinterpret_cast<uint16_t*>(cache.v + place + (int64_t)kv * cache.page * (D * 2)), plain, x[i]);
      }
    }
  }
}

// ---- rows to pages of e4m3 -----------------------------------------------------------------------
__device__ __forceinline__ float finite_magnitude(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;                     // NaN compares false
}
// smallest 2^e, e >= -120, with a <= 448 * 2^e
__device__ __forceinline__ float scale_for(float a) {
  const uint32_t u = __float_as_uint(a);
  int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);     // 448 = 1.75 * 2^8
  e = e > kMinScaleExponent ? e : kMinScaleExponent;
  return __uint_as_float((uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ float as_e4m3_range(float x) {
  // beyond the largest value only what is infinite or NaN: both become NaN
  return fabsf(x) < INFINITY ? fminf(fmaxf(x, -kE4m3Max), kE4m3Max) : NAN;
}
__device__ __forceinline__ uint32_t e4m3_quad(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(as_e4m3_range(a), as_e4m3_range(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(as_e4m3_range(c), as_e4m3_range(d), w, true);
  return (uint32_t)w;
}

// One workgroup for a page that a sequence appends to, a kv head, and K (z = 0) or V; kItems units a thread cover a page, and
// stay in registers between the maximum and the rounding.  Sequence s has the slots from start / page + 2 s: n tokens touch at
// most n / page + 2 pages.
template <int D, int kItems>
__global__ __launch_bounds__(256) void append_e4m3_kernel(Rows k_in, Rows v_in, RotaryTable rot, CacheView cache,
                                                          BatchView batch) {
  constexpr int U = D / 16;
  __shared__ float s_max[4];
  const int s = __builtin_amdgcn_readfirstlane(seq_at(batch, blockIdx.x, 1, cache.page_shift, 2));
  const SeqRows r = seq_rows(batch, s);
  const int start = r.length - r.n, start0 = max(start, 0);
  const int64_t page64 = (int64_t)(start0 >> cache.page_shift) + (int)blockIdx.x - ((r.row0 >> cache.page_shift) + 2 * s);
  if (r.n == 0 || page64 < 0 || page64 >= batch.max_pages || page64 * cache.page >= r.length) return;
  const int page = (int)page64, first = page << cache.page_shift;
  const int begin = max(start0 - first, 0), end = min(r.length - first, cache.page);     // places of the new tokens
  const int id = batch.table[(int64_t)s * batch.max_pages + page];
  if (id < 0 || id >= cache.n_pages || begin >= end) return;
  const int kv = blockIdx.y, t = threadIdx.x, u = t % U;
  const bool is_k = blockIdx.z == 0;
  const Rows in = is_k ? k_in : v_in;
  char* dst = (is_k ? cache.k : cache.v) + id * cache.page_stride + (int64_t)kv * cache.page * D;
  float* scale_at = (is_k ? cache.k_scale : cache.v_scale) + (int64_t)id * cache.h_kv + kv;
  const float old = begin > 0 ? *scale_at : 0.f;
  const uint16_t* src = in.p + kv * in.head + (int64_t)(r.row0 + first - start) * in.token;    // row of place 0
  const Places at = is_k ? places_of(rot, u) : Places{16 * u, 16 * u + 8, false};

  Unit raw[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int row = begin + t / U + i * (256 / U);
    raw[i] = Unit{make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
    if (row < end) raw[i] = load_unit(src + row * in.token, at);
  }
  float x[kItems][16], top = 0.f;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int row = begin + t / U + i * (256 / U);
    Turn turn = {};
    if (at.turns && row < end) turn = turn_of(rot, u, (double)(first + row));
    turned_values(rot, raw[i], at.turns, turn, x[i]);
#pragma unroll
    for (int j = 0; j < 16; ++j) top = fmaxf(top, finite_magnitude(x[i][j]));
  }
  top = wave_max(top);
  if ((t & 63) == 0) s_max[t >> 6] = top;
  __syncthreads();                                   // and everyone has read the old scale
  top = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  const float need = scale_for(top);
  const float scale = begin > 0 && old > need ? old : need;
  if (t == 0) *scale_at = scale;
  if (begin > 0 && scale > old) {                    // what is there moves with the scale
    const float by = old / scale;
    for (int i = t; i < begin * (D / 4); i += 256) {
      uint32_t* w = reinterpret_cast<uint32_t*>(dst) + i;
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)*w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)*w, true);
      *w = e4m3_quad(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
    }
  }
  // a power of two, unless the page came with another scale: x / scale is x * (1 / scale) then, exactly
  const bool exact = (__float_as_uint(scale) & 0x7FFFFFu) == 0;
  const float by = 1.f / scale;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int row = begin + t / U + i * (256 / U);
    if (row >= end) break;
#pragma unroll
    for (int j = 0; j < 16; ++j) x[i][j] = exact ? x[i][j] * by : x[i][j] / scale;
    char* d = dst + row * D;
    *reinterpret_cast<uint2*>(d + at.a) = make_uint2(e4m3_quad(x[i][0], x[i][1], x[i][2], x[i][3]), e4m3_quad(x[i][4], x[i][5], x[i][6], x[i][7]));
    *reinterpret_cast<uint2*>(d + at.b) = make_uint2(e4m3_quad(x[i][8], x[i][9], x[i][10], x[i][11]), e4m3_quad(x[i][12], x[i][13], x[i][14], x[i][15]));
  }
}

template <int D, bool kPaged>
static int launch_rows(const RowJob& job, const RotaryTable& rot, const int32_t* positions, const CacheView& cache,
                       const BatchView& batch, hipStream_t st) {
  const int heads = job.n_q + job.n_k + job.n_v;
  if (heads == 0) return PRISM_OK;
  const int64_t units = (int64_t)job.n_tokens * (D / 16);
  // Four heads a thread, so that the angles of a unit are formed once for them; in calls that do not fill the chip one, so that no
  // head waits for another.  us at 1 / 2 / 4 / 8 heads a thread: 32768 tokens of 28/4 heads 127.6 / 100.8 / 99.4 / 101.7, 20011
  // of 32/8 inside a projection 143.5 / 108.6 / 99.4 / 96.6, 32768 of 8 appended as they are 59.6 / 57.9 / 59.5 / 62.8; the kernel of 1
  // token of 32/8 4.6 with one head, 5.9 with four.
  const int each = units * heads <= 1 << 17 ? 1 : 4;
  // Neighbouring workgroups go on where the inputs do: us with the next tokens / with the next heads, heads inside a projection (20011
  // tokens of 32/8 heads) 99.3 / 88.2, dense tensors (32768 of 28/4) 99.1 / 106.4, (32768 of 8, appended) 59.6 / 63.9.
  const Rows& in = job.n_q > 0 ? job.q_in : job.k_in;
  const unsigned blocks = (unsigned)((units + 255) / 256), groups = (heads + each - 1) / each;
  const bool heads_first = in.head < in.token && blocks < 65536;
  hipLaunchKernelGGL((rows_kernel<D, kPaged>), heads_first ? dim3(groups, blocks) : dim3(blocks, groups), dim3(256), 0, st, job, rot,
                     positions, cache, batch, each, heads_first ? 1 : 0);
  return launch_status();
}
template <bool kPaged>
static int launch_rows_for(int d, const RowJob& job, const RotaryTable& rot, const int32_t* positions, const CacheView& cache,
                           const BatchView& batch, hipStream_t st) {
  switch (d) {
    case 64: return launch_rows<64, kPaged>(job, rot, positions, cache, batch, st);
    case 128: return launch_rows<128, kPaged>(job, rot, positions, cache, batch, st);
    default: return launch_rows<256, kPaged>(job, rot, positions, cache, batch, st);
  }
}
template <int D>
static int launch_append_e4m3(const Rows& k, const Rows& v, const RotaryTable& rot, const CacheView& cache,
                              const BatchView& batch, hipStream_t st) {
  const dim3 grid((unsigned)(batch.n_tokens >> cache.page_shift) + 2 * (unsigned)batch.n_seqs, cache.h_kv, 2);
  switch (cache.page * (D / 16) / 256) {
    case 0: case 1: hipLaunchKernelGGL((append_e4m3_kernel<D, 1>), grid, dim3(256), 0, st, k, v, rot, cache, batch); break;
    case 2: hipLaunchKernelGGL((append_e4m3_kernel<D, 2>), grid, dim3(256), 0, st, k, v, rot, cache, batch); break;
    case 4: hipLaunchKernelGGL((append_e4m3_kernel<D, 4>), grid, dim3(256), 0, st, k, v, rot, cache, batch); break;
    default: hipLaunchKernelGGL((append_e4m3_kernel<D, 8>), grid, dim3(256), 0, st, k, v, rot, cache, batch); break;
  }
  return launch_status();
}

}  // namespace prism

using namespace prism;

extern "C" int prism_rotate(const prism_rotary* rotary, int head_dim, int n_tokens, const int32_t* positions,
                            int n_q_heads, const prism_rows* q_in, const prism_rows* q_out, int n_kv_heads,
                            const prism_rows* k_in, const prism_rows* k_out, uint32_t flags, void* stream) {
  if (!known_head_dim(head_dim)) return PRISM_ERR_UNSUPPORTED;
  int rc = check_rotary(rotary, head_dim);
  if (rc != PRISM_OK) return rc;
  if (n_tokens < 0 || n_q_heads < 0 || n_kv_heads < 0 || (flags & ~PRISM_ROTATE_BACKWARD) != 0) return PRISM_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens || n_q_heads > kMaxHeads || n_kv_heads > kMaxHeads) return PRISM_ERR_UNSUPPORTED;
  if (n_tokens == 0) return PRISM_OK;
  struct { const prism_rows *in, *out; int heads; } sides[2] = {{q_in, q_out, n_q_heads}, {k_in, k_out, n_kv_heads}};
  for (const auto& s : sides) {
    if (s.heads == 0) continue;
    if ((rc = check_rows(s.in, s.heads, n_tokens, head_dim, false)) != PRISM_OK ||
        (rc = check_rows(s.out, s.heads, n_tokens, head_dim, true)) != PRISM_OK ||
        (rc = check_in_place(s.in, s.out, s.heads, n_tokens)) != PRISM_OK)
      return rc;
  }
  const RowJob job = {rows_of(q_in), rows_of(q_out), rows_of(k_in), rows_of(k_out), Rows{}, n_q_heads, n_kv_heads, 0, n_tokens};
  return launch_rows_for<false>(head_dim, job, rotary_table(rotary, (flags & PRISM_ROTATE_BACKWARD) != 0), positions, CacheView{},
                                BatchView{}, static_cast<hipStream_t>(stream));
}

extern "C" int prism_cache_append(const prism_cache* cache, const prism_batch* batch, const prism_rotary* rotary,
                                  const prism_rows* k, const prism_rows* v, int n_q_heads, const prism_rows* q_in,
                                  const prism_rows* q_out, void* stream) {
  int rc = check_cache(cache);
  if (rc != PRISM_OK || (rc = check_batch(cache, batch)) != PRISM_OK) return rc;
  const int d = cache->head_dim, T = batch->n_tokens, h_kv = cache->n_kv_heads;
  if (rotary != nullptr && (rc = check_rotary(rotary, d)) != PRISM_OK) return rc;
  const bool with_q = q_in != nullptr || q_out != nullptr;
  if (n_q_heads < 0 || (with_q && n_q_heads == 0)) return PRISM_ERR_INVALID_ARG;
  if (n_q_heads > kMaxHeads) return PRISM_ERR_UNSUPPORTED;
  if (T == 0) return PRISM_OK;
  if ((rc = check_cache_memory(cache)) != PRISM_OK || (rc = check_rows(k, h_kv, T, d, false)) != PRISM_OK ||
      (rc = check_rows(v, h_kv, T, d, false)) != PRISM_OK)
    return rc;
  if (with_q && ((rc = check_rows(q_in, n_q_heads, T, d, false)) != PRISM_OK ||
                 (rc = check_rows(q_out, n_q_heads, T, d, true)) != PRISM_OK ||
                 (rc = check_in_place(q_in, q_out, n_q_heads, T)) != PRISM_OK))
    return rc;
  const CacheView c = cache_view(cache);
  const BatchView b = batch_view(batch);
  const RotaryTable rot = rotary_table(rotary, false);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->dtype == PRISM_CACHE_E4M3;
  const int heads = e4m3 ? 0 : h_kv;
  const RowJob job = {rows_of(q_in), rows_of(q_out), rows_of(k), Rows{}, rows_of(v), with_q ? n_q_heads : 0, heads, heads, T};
  rc = launch_rows_for<true>(d, job, rot, nullptr, c, b, st);
  if (rc != PRISM_OK || !e4m3) return rc;
  switch (d) {
    case 64: return launch_append_e4m3<64>(rows_of(k), rows_of(v), rot, c, b, st);
    case 128: return launch_append_e4m3<128>(rows_of(k), rows_of(v), rot, c, b, st);
    default: return launch_append_e4m3<256>(rows_of(k), rows_of(v), rot, c, b, st);
  }
}
