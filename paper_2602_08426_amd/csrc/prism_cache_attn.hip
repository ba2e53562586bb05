// Attention of new tokens over the paged cache (gfx950): prism_cache_attn.
//
// The rows of a (sequence, kv head) are its new tokens times the q-heads of the kv head: row r = token r / g, head r % g,
// so that a tile of keys and values is read once for all of them.
#include "prism_cache.h"
#include "prism_tiles.h"

#include <type_traits>

namespace prism {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// a value that is the same in all lanes, in a scalar register
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// Infinities and NaN among packed values: the top bits of theirs (bf16: an exponent of ones; e4m3: NaN, 0x7F and 0xFF), and the
// word with zeros in their place.
template <bool kE4m3>
__device__ __forceinline__ uint32_t special_bits(uint32_t w) {
  return kE4m3 ? ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u : ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}
template <bool kE4m3>
__device__ __forceinline__ uint32_t without_specials(uint32_t w) {
  const uint32_t n = special_bits<kE4m3>(w);
  return w & ~(kE4m3 ? (n >> 7) * 0xFFu : (n >> 15) * 0xFFFFu);
}

// eight e4m3 values times a power of two as bf16
__device__ __forceinline__ u32x4 bf16_of_e4m3(uint32_t lo, uint32_t hi, float power) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, true))};
}

// What the kernels need to know of a call.
struct AttnCall {
  Rows q, out;
  float* lse;
  CacheView cache;
  BatchView batch;         // each = max_tokens
  int h, g;                // q-heads, of a kv head
  int window, sinks;
  float scale;             // of the scores, times log2(e)
  int step_rows;           // a sequence and kv head of at most so many rows is step_kernel's, others chunk_kernel's
};

// The keys that some row of a sequence (or of a part of its new tokens) sees, in tiles of kTile tokens: the tiles [0, sink)
// and [low, end).
struct KeyRange {
  int sink, low, end;
  __device__ __forceinline__ int count() const { return sink + end - low; }
  __device__ __forceinline__ int tile(int i) const { return i < sink ? i : low + i - sink; }
};
template <int kTile>
__device__ __forceinline__ KeyRange key_range(const AttnCall& a, int first_pos, int last_pos) {
  const int keys = min(last_pos + 1, a.batch.max_pages << a.cache.page_shift);
  KeyRange k = {0, 0, 0};
  if (keys <= 0) return k;
  k.end = (keys + kTile - 1) / kTile;
  if (a.window > 0) {
    k.low = min(max(first_pos - a.window + 1, 0) / kTile, k.end);
    k.sink = min((min(a.sinks, keys) + kTile - 1) / kTile, k.low);
  }
  return k;
}

// =====================================================================================
// Steps: few rows per sequence and kv head (up to 16 * MT), bound by the bytes of the cache.
//
// Work.  A unit is four tiles of 32 keys of one (sequence, kv head), one tile for each wave of a workgroup.  The units of all
// sequences and kv heads, one behind the other, are dealt to the workgroups in equal shares, whatever the lengths are: share
// w of W is [w * total / W, (w + 1) * total / W).  A workgroup that has all units of a (sequence, kv head) writes its
// output; otherwise each of those that have a part leaves its unscaled sums, and combine_kernel joins them.  Nothing
// depends on which workgroup runs when.
//
// A wave keeps everything in registers: no tile passes through LDS.  16x16x32 MFMAs on the transposed problem,
//     S^T = K Q^T     A = 16 keys (lane m = l%16 holds key 8*(m/4) + 4*t + m%4 of the tile, t the MFMA), B = rows of Q
//     O^T += V^T P^T  A = 16 dims, 32 keys (lane: keys 8*(l/16) + j), B = P^T
// With the keys of S^T ordered like that, lane l holds the scores of row l%16 with keys 8*(l/16) + j, which is the B operand of
// the second product.  A operand of V^T: a lane loads whole pieces of 8 token rows and pairs up their halves (v_perm), which
// transposes 8 x 8 values inside the lane.  The dims of a k-step of S^T are any, as long as Q has the same: a lane's are where its
// 16-byte pieces lie.  P is rounded to bf16 for the second product, 2^-8 of a probability at most; sums and maxima are fp32.
//
// Measured, d = 128 (kernel alone): 64 sequences of 500 to 32000 tokens, 32/8 heads, 2.06 GB of bf16 keys and values, 349 us = 5.9
// TB/s; 8 of 128K, e4m3, 2.08 GB, 349 us = 6.0 TB/s; 16 with a window of 4096, 28/4 heads, 135 MB, 26 us = 5.2 TB/s.  A large copy
// on this card moves 5.0 TB/s, reading alone 5.7 to 6.9; the counters show the cache's bytes read once and the matrix
// cores busy for 4 to 8 % of the time.  One sequence of 2048 is the latency of a unit, 8 us.
// =====================================================================================
constexpr int kTile = 32, kStepWaves = 4;
constexpr int kStepThreads = kStepWaves * 64;

__device__ __forceinline__ KeyRange keys_of(const AttnCall& a, const SeqRows& r) {
  const int n = min(r.n, a.batch.each);
  if (n == 0 || (int64_t)n * a.g > a.step_rows) return KeyRange{0, 0, 0};
  return key_range<kTile>(a, r.length - r.n, r.length - r.n + n - 1);
}

// Prefix sums over the units of all sequences, 256 at a time.
struct StepScan {
  int before[kStepThreads + 1];      // units of the sequences in front, within these 256
  int part[kStepWaves];
  SeqRows rows[kStepThreads];
};
// all threads; returns the units of sequences s0 .. s0 + 255
__device__ __forceinline__ int scan_units(StepScan& m, const AttnCall& a, int s0) {
  const int t = threadIdx.x, wave = t >> 6;
  const SeqRows r = s0 + t < a.batch.n_seqs ? seq_rows(a.batch, s0 + t) : SeqRows{0, 0, 0};
  const int upto = wave_scan_inclusive((keys_of(a, r).count() + kStepWaves - 1) / kStepWaves);
  __syncthreads();
  m.rows[t] = r;
  if ((t & 63) == 63) m.part[wave] = upto;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < kStepWaves; ++w) base += w < wave ? m.part[w] : 0;
  m.before[t + 1] = base + upto;
  if (t == 0) m.before[0] = 0;
  __syncthreads();
  return uniform(m.before[kStepThreads]);
}

// Shares that are dealt: none is empty, so that the parts of a (sequence, kv head) lie in consecutive ones.
__device__ __forceinline__ int64_t shares(int64_t total, int workgroups) { return total < workgroups ? total : workgroups; }

struct StepWs {
  float* part;             // [2 * workers][16 * MT][D] unscaled sums
  float2* stats;           // [2 * workers][16 * MT] maximum (in units of log2) and sum
};

template <int D, bool kE4m3>
struct StepCfg {
  static constexpr int kElem = kE4m3 ? 1 : 2;
  static constexpr int kKSteps = D / 32;
  static constexpr int kKLoads = 2 * D * kElem / 64;      // 16-byte pieces a lane takes of a K tile
  static constexpr int kVWords = D / 16 * kElem / 4;      // words a lane takes of a V row
  static constexpr int kDTiles = D / 16;
};

// V pieces of a lane: dims (i / 8) * 128 + 8 m + i % 8 of D = 256, (D / 16) m + i otherwise
template <int D>
__device__ __forceinline__ int lane_dim(int m, int i) {
  return D == 256 ? (i >> 3) * 128 + 8 * m + (i & 7) : (D / 16) * m + i;
}

template <int D, bool kE4m3, int MT>
__global__ __launch_bounds__(kStepThreads, D == 256 || (MT > 1 && !kE4m3) ? 1 : 2) void step_kernel(AttnCall a, StepWs ws) {
#if defined(__HIP_DEVICE_COMPILE__)
  using C = StepCfg<D, kE4m3>;
  constexpr int kRow = D * C::kElem;                      // bytes of a token's row
  constexpr int kPad = D + 4;
  __shared__ StepScan scan;
  __shared__ float s_stats[2][kStepWaves][16];
  __shared__ float s_o[kStepWaves][16][kPad];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int m = lane & 15, qd = lane >> 4;
  const int h_kv = a.cache.h_kv;

  int64_t total = 0;
  int chunk_units = 0;
  for (int s0 = 0; s0 < a.batch.n_seqs; s0 += kStepThreads) {
    chunk_units = scan_units(scan, a, s0);
    total += chunk_units;
  }
  total *= h_kv;
  const int64_t W = shares(total, gridDim.x);
  const int64_t from = total * blockIdx.x / W, to = total * (blockIdx.x + 1) / W;
  if (blockIdx.x >= W) return;

  // offsets of this lane's pieces of a tile
  int k_off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) k_off[i] = (8 * (m >> 2) + 4 * i + (m & 3)) * kRow + qd * 16;
  const int v_off = 8 * qd * kRow + (D == 256 && !kE4m3 ? m * 16 : (kE4m3 && D == 256 ? m * 8 : m * (kRow / 16)));

  int64_t chunk0 = 0;                                     // first unit of the 256 sequences
  for (int s0 = 0; s0 < a.batch.n_seqs && chunk0 < to; s0 += kStepThreads) {
    if (a.batch.n_seqs > kStepThreads) chunk_units = scan_units(scan, a, s0);
    const int64_t chunk1 = chunk0 + (int64_t)chunk_units * h_kv;
    int64_t at = from > chunk0 ? from : chunk0;
    const int64_t stop = to < chunk1 ? to : chunk1;
    int i = 0;
    if (at < stop) {                                      // the sequence of the first unit
      const int want = (int)((at - chunk0) / h_kv);
      int lo = 0, hi = kStepThreads;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (scan.before[mid] <= want) lo = mid; else hi = mid;
      }
      i = uniform(lo);
    }
    for (; at < stop; ++i) {
      const int before = uniform(scan.before[i]), units = uniform(scan.before[i + 1]) - before;
      if (units == 0) continue;
      const int64_t seq_first = chunk0 + (int64_t)before * h_kv;
      const int64_t seq_end = seq_first + (int64_t)units * h_kv;
      const int s = s0 + i;
      const SeqRows r = {uniform(scan.rows[i].row0), uniform(scan.rows[i].n), uniform(scan.rows[i].length)};
      const KeyRange keys = keys_of(a, r);
      const int n = min(r.n, a.batch.each), R = n * a.g;
      const int pos0 = r.length - r.n, pos_last = pos0 + n - 1;
      const int32_t* table = a.batch.table + (int64_t)s * a.batch.max_pages;
      while (at < stop && at < seq_end) {
        const int kv = (int)((at - seq_first) / units);
        const int64_t item_first = seq_first + (int64_t)kv * units, item_end = item_first + units;
        const int u0 = (int)(at - item_first), u1 = (int)((stop < item_end ? stop : item_end) - item_first);
        at = item_first + u1;

        // ---- rows of Q: B operands ----
        bf16x8 qf[MT][C::kKSteps];
        int row_pos[MT];
#pragma unroll
        for (int x = 0; x < MT; ++x) {
          const int row = min(16 * x + m, R - 1), tok = row / a.g;
          row_pos[x] = pos0 + tok;
          const uint16_t* qp = a.q.p + (int64_t)(kv * a.g + row - tok * a.g) * a.q.head + (int64_t)(r.row0 + tok) * a.q.token;
#pragma unroll
          for (int ks = 0; ks < C::kKSteps; ++ks)
            qf[x][ks] = *reinterpret_cast<const bf16x8*>(qp + (kE4m3 ? (ks >> 1) * 64 + qd * 16 + (ks & 1) * 8 : ks * 32 + qd * 8));
        }

        f32x4 o[MT][C::kDTiles];
        float m_run[MT], l_run[MT];
#pragma unroll
        for (int x = 0; x < MT; ++x) {
          m_run[x] = -INFINITY;
          l_run[x] = 0.f;
#pragma unroll
          for (int d = 0; d < C::kDTiles; ++d) o[x][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        // ---- the wave's tiles: entries of the page table (and scales) held 64 a time, one a lane ----
        int held_from = 0, held = 0;
        float held_ks = 0.f, held_vs = 0.f;
        auto hold = [&](int from_entry) __attribute__((always_inline)) {
          held_from = from_entry;
          const int e = from_entry + lane;
          held = e < a.batch.max_pages ? table[e] : -1;
          if (held >= a.cache.n_pages) held = -1;
          if (kE4m3) {
            const int64_t sc = (int64_t)max(held, 0) * h_kv + kv;
            held_ks = a.cache.k_scale[sc];
            held_vs = a.cache.v_scale[sc];
          }
        };
        struct TileAt {
          int tile, page;                                 // page < 0: none
          float ks, vs;
          int64_t off;                                    // of the tile in k and in v, and its bytes
          int bytes;
        };
        auto locate = [&](int list_at) __attribute__((always_inline)) {
          TileAt x;
          x.tile = keys.tile(list_at);
          const int tok = x.tile * kTile, e = tok >> a.cache.page_shift;
          if ((unsigned)(e - held_from) >= 64u) hold(e);
          x.page = __builtin_amdgcn_readlane(held, e - held_from);
          if (kE4m3) {
            x.ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, held_ks), e - held_from));
            x.vs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, held_vs), e - held_from));
          }
          x.off = max(x.page, 0) * a.cache.page_stride + (int64_t)(kv * a.cache.page + (tok & (a.cache.page - 1))) * kRow;
          x.bytes = x.page < 0 ? 0 : min(kTile, r.length - tok) * kRow;           // what lies behind the last token reads as zero
          return x;
        };
        u32x4 kw[C::kKLoads];
        uint32_t vw[8][C::kVWords];
        // the descriptors are formed here, from scalars: kept in a TileAt they went through memory at D = 256, and a loop over the
        // lanes' different values stood around each load
        auto load_k = [&](const TileAt& x) __attribute__((always_inline)) {
          const __amdgpu_buffer_rsrc_t from = make_rsrc(a.cache.k + uniform(x.off), uniform(x.bytes));
#pragma unroll
          for (int j = 0; j < C::kKLoads; ++j)
            kw[j] = __builtin_amdgcn_raw_buffer_load_b128(from, k_off[j / (C::kKLoads / 2)] + (j % (C::kKLoads / 2)) * 64, 0, 0);
        };
        auto load_v = [&](const TileAt& x) __attribute__((always_inline)) {
          const __amdgpu_buffer_rsrc_t from = make_rsrc(a.cache.v + uniform(x.off), uniform(x.bytes));
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if constexpr (C::kVWords == 1) {
              vw[j][0] = __builtin_amdgcn_raw_buffer_load_b32(from, v_off + j * kRow, 0, 0);
            } else if constexpr (C::kVWords == 2) {
              const auto w = __builtin_amdgcn_raw_buffer_load_b64(from, v_off + j * kRow, 0, 0);
              vw[j][0] = w[0];
              vw[j][1] = w[1];
            } else if constexpr (kE4m3) {                 // D = 256: two halves of 128 dims
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                const auto w = __builtin_amdgcn_raw_buffer_load_b64(from, v_off + j * kRow + hf * 128, 0, 0);
                vw[j][2 * hf] = w[0];
                vw[j][2 * hf + 1] = w[1];
              }
            } else {
#pragma unroll
              for (int hf = 0; hf < C::kVWords / 4; ++hf) {
                const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(from, v_off + j * kRow + hf * 256, 0, 0);
                vw[j][4 * hf] = w[0];
                vw[j][4 * hf + 1] = w[1];
                vw[j][4 * hf + 2] = w[2];
                vw[j][4 * hf + 3] = w[3];
              }
            }
          }
        };
        // A operand of a k-step of S^T
        auto k_frag = [&](int i, int ks) __attribute__((always_inline)) {
          if constexpr (!kE4m3) {
            return __builtin_bit_cast(bf16x8, kw[i * C::kKSteps + ks]);
          } else {
            const u32x4 w = kw[i * (C::kKSteps / 2) + (ks >> 1)];
            bf16x8 f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * (ks & 1) + e], 1.0f, false);
              const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * (ks & 1) + e], 1.0f, true);
              f[4 * e] = lo[0]; f[4 * e + 1] = lo[1]; f[4 * e + 2] = hi[0]; f[4 * e + 3] = hi[1];
            }
            return f;
          }
        };
        // A operand of O^T, dims lane_dim(., d): the lane's 8 keys of that dim
        auto v_frag = [&](int d) __attribute__((always_inline)) {
          u32x4 w;
#pragma unroll
          for (int p = 0; p < 4; ++p) {                   // keys 2p, 2p + 1
            if constexpr (!kE4m3) {
              w[p] = __builtin_amdgcn_perm(vw[2 * p + 1][d >> 1], vw[2 * p][d >> 1], (d & 1) ? 0x07060302u : 0x05040100u);
            } else {
              const uint32_t b = __builtin_amdgcn_perm(vw[2 * p + 1][d >> 2], vw[2 * p][d >> 2], (d & 2) ? 0x07030602u : 0x05010400u);
              const bf16x2 y = (d & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true)
                                       : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
              w[p] = __builtin_bit_cast(uint32_t, y);
            }
          }
          return __builtin_bit_cast(bf16x8, w);
        };

        const int list_end = min(u1 * kStepWaves, keys.count());
        int list_at = u0 * kStepWaves + wave;
        TileAt now = {}, next = {};
        if (list_at < list_end) {
          hold((keys.tile(list_at) * kTile) >> a.cache.page_shift);
          now = locate(list_at);
          load_k(now);
          load_v(now);
        }
        for (; list_at < list_end; list_at += kStepWaves) {
          const bool more = list_at + kStepWaves < list_end;
          if (more) next = locate(list_at + kStepWaves);

          // ---- S^T = K Q^T ----
          f32x4 sc[MT][2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int ks = 0; ks < C::kKSteps; ++ks) {
              const bf16x8 f = k_frag(i, ks);
#pragma unroll
              for (int x = 0; x < MT; ++x)
                sc[x][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf[x][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[x][i], 0, 0, 0);
            }
          }
          if (more) load_k(next);

          // ---- which keys a row sees: all of the tile, or each for itself ----
          const int first = now.tile * kTile, last = first + kTile - 1;
          const bool whole = now.page >= 0 && last <= pos0 && (a.window == 0 || first > pos_last - a.window || last < a.sinks);
          // Without branches: from && and || the compiler (AMD clang 22) made control flow around the writes of single score
          // elements, and lost one of them.
          const int window = a.window > 0 ? a.window : 0x40000000;
          auto sees = [&](int key, int pos) __attribute__((always_inline)) {
            return (now.page >= 0) & (key <= pos) & ((key > pos - window) | (key < a.sinks));
          };
          bool special = false;
          if (!whole) {
#pragma unroll
            for (int x = 0; x < MT; ++x)
#pragma unroll
              for (int j = 0; j < 8; ++j)
                sc[x][j >> 2][j & 3] = sees(first + 8 * qd + j, row_pos[x]) ? sc[x][j >> 2][j & 3] : -INFINITY;
            // 0 * NaN is NaN: infinities and NaN among the values leave the product and are added where they are seen
            uint32_t bad = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int w = 0; w < C::kVWords; ++w) bad |= special_bits<kE4m3>(vw[j][w]);
            special = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
            if (special) {
#pragma unroll
              for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 0; w < C::kVWords; ++w) vw[j][w] = without_specials<kE4m3>(vw[j][w]);
            }
          }

          // ---- online softmax: a row is in the lanes m, m + 16, m + 32, m + 48 ----
          bf16x8 pf[MT];
          const float by = kE4m3 ? a.scale * now.ks : a.scale;
#pragma unroll
          for (int x = 0; x < MT; ++x) {
            float mx = fmaxf(fmaxf(fmaxf(sc[x][0][0], sc[x][0][1]), fmaxf(sc[x][0][2], sc[x][0][3])),
                             fmaxf(fmaxf(sc[x][1][0], sc[x][1][1]), fmaxf(sc[x][1][2], sc[x][1][3])));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m_run[x], mx * by);
            if (__builtin_amdgcn_ballot_w64(m_new > m_run[x]) != 0) {     // some row's maximum moved
              const float keep = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[x] - m_new);
              l_run[x] *= keep;
#pragma unroll
              for (int d = 0; d < C::kDTiles; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[x][d][e] *= keep;
              m_run[x] = m_new;
            }
            const float base = m_new == -INFINITY ? 0.f : m_new;          // nothing seen yet: all p are 0
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
              float p0 = __builtin_amdgcn_exp2f(fmaf(sc[x][j >> 2][j & 3], by, -base));
              float p1 = __builtin_amdgcn_exp2f(fmaf(sc[x][j >> 2][(j & 3) + 1], by, -base));
              l_run[x] += p0 + p1;
              if (kE4m3) {
                p0 *= now.vs;
                p1 *= now.vs;
              }
              const f32x2 pp = {p0, p1};
              const bf16x2 pb = __builtin_convertvector(pp, bf16x2);
              pf[x][j] = pb[0];
              pf[x][j + 1] = pb[1];
            }
          }

          // ---- O^T += V^T P^T ----
#pragma unroll
          for (int d = 0; d < C::kDTiles; ++d) {
            const bf16x8 f = v_frag(d);
#pragma unroll
            for (int x = 0; x < MT; ++x) o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pf[x], o[x][d], 0, 0, 0);
          }
          if (special) {
            // p > 0 times an infinity or NaN is that
            const int there = now.page < 0 ? 0 : min(kTile, r.length - first);
            const char* vp = a.cache.v + max(now.page, 0) * a.cache.page_stride + (int64_t)(kv * a.cache.page + (first & (a.cache.page - 1))) * kRow;
#pragma unroll 1
            for (int j = 0; j < there; ++j)
#pragma unroll
              for (int d = 0; d < C::kDTiles; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const char* vq = vp + j * kRow + lane_dim<D>(4 * qd + e, d) * C::kElem;
                  float y;
                  if constexpr (kE4m3)
                    y = __builtin_amdgcn_cvt_f32_fp8(*reinterpret_cast<const uint8_t*>(vq), 0);
                  else
                    y = bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(vq));
                  const bool odd = !(fabsf(y) < INFINITY);
#pragma unroll
                  for (int x = 0; x < MT; ++x) o[x][d][e] = odd & sees(first + j, row_pos[x]) ? o[x][d][e] + y : o[x][d][e];
                }
          }
          if (more) {
            load_v(next);
            now = next;
          }
        }

        // ---- the four waves' sums; to the output, or left for combine_kernel ----
        const bool all = u0 == 0 && u1 == units;
        const int slot = 2 * blockIdx.x + (u0 == 0 ? 1 : 0);
#pragma unroll
        for (int x = 0; x < MT; ++x) {
          float l = l_run[x];
          l += __shfl_xor(l, 16);
          l += __shfl_xor(l, 32);
          __syncthreads();                                // the tile before has been read
          if (qd == 0) {
            s_stats[0][wave][m] = m_run[x];
            s_stats[1][wave][m] = l;
          }
#pragma unroll
          for (int d = 0; d < C::kDTiles; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_o[wave][m][lane_dim<D>(4 * qd + e, d)] = o[x][d][e];
          __syncthreads();
          constexpr int kEach = D / 16;                   // dims of a thread
          const int row16 = t >> 4, d0 = (t & 15) * kEach, row = 16 * x + row16;
          if (row >= R) continue;
          float top = s_stats[0][0][row16];
#pragma unroll
          for (int w = 1; w < kStepWaves; ++w) top = fmaxf(top, s_stats[0][w][row16]);
          const float base = top == -INFINITY ? 0.f : top;
          float sum = 0.f, acc[kEach];
#pragma unroll
          for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
#pragma unroll
          for (int w = 0; w < kStepWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_stats[0][w][row16] - base);
            sum += f * s_stats[1][w][row16];
#pragma unroll
            for (int e = 0; e < kEach; ++e) acc[e] += f * s_o[w][row16][d0 + e];
          }
          if (all) {
            const int tok = row / a.g, hq = kv * a.g + row - tok * a.g;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            uint16_t* op = a.out.p + (int64_t)hq * a.out.head + (int64_t)(r.row0 + tok) * a.out.token + d0;
#pragma unroll
            for (int e = 0; e < kEach; e += 4)
              *reinterpret_cast<uint2*>(op + e) = make_uint2(bf16_pair(acc[e] * inv, acc[e + 1] * inv), bf16_pair(acc[e + 2] * inv, acc[e + 3] * inv));
            if (a.lse != nullptr && (t & 15) == 0)
              a.lse[(int64_t)hq * a.batch.n_tokens + r.row0 + tok] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
          } else {
            float* pp = ws.part + ((int64_t)slot * (16 * MT) + row) * D + d0;
#pragma unroll
            for (int e = 0; e < kEach; e += 4) *reinterpret_cast<float4*>(pp + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
            if ((t & 15) == 0) ws.stats[(int64_t)slot * (16 * MT) + row] = make_float2(top, sum);
          }
        }
      }
    }
    chunk0 = chunk1;
  }
#endif
}

// Joins the parts of a row that several workgroups of step_kernel worked on, and writes the rows of sequences in which no row
// sees anything.  One workgroup a row; kGroups groups of threads take every kGroups-th part, each with a maximum of its own, so
// that all parts are requested at once.  Bound by latency: 3 to 7 us, of which a kernel that does nothing has 3.6 in a queue.
template <int D, int MT>
__global__ __launch_bounds__(kStepThreads) void combine_kernel(AttnCall a, StepWs ws, int workgroups) {
  constexpr int kGroups = kStepThreads * 4 / D;
  __shared__ StepScan scan;
  __shared__ float s_acc[kGroups][D];
  __shared__ float s_top[kGroups], s_sum[kGroups];
  const int s = blockIdx.x, kv = blockIdx.y, row = blockIdx.z, t = threadIdx.x, h_kv = a.cache.h_kv;
  const SeqRows r = seq_rows(a.batch, s);
  const int64_t rows = (int64_t)min(r.n, a.batch.each) * a.g;
  if (row >= rows || rows > a.step_rows) return;
  int64_t total = 0, first = 0;
  int units = 0;
  for (int s0 = 0; s0 < a.batch.n_seqs; s0 += kStepThreads) {
    const int all = scan_units(scan, a, s0);
    if (s >= s0 && s < s0 + kStepThreads) {
      units = scan.before[s - s0 + 1] - scan.before[s - s0];
      first = (total + scan.before[s - s0]) * h_kv + (int64_t)kv * units;
    }
    total += all;
  }
  total *= h_kv;
  const int64_t W = shares(total, workgroups);
  // the workgroup of unit x: the largest w with w * total / W <= x
  const int w0 = units > 0 ? (int)(((first + 1) * W - 1) / total) : 0;
  const int w1 = units > 0 ? (int)(((first + units) * W - 1) / total) : 0;
  if (units > 0 && w0 == w1) return;
  const int group = t / (D / 4), d0 = t % (D / 4) * 4;
  float top = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (units > 0) {
    constexpr int kAtOnce = 4;
    for (int w = w0 + group; w <= w1; w += kAtOnce * kGroups) {
      float2 st[kAtOnce];
      float4 x[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int wi = w + i * kGroups;
        st[i] = make_float2(-INFINITY, 0.f);
        x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (wi <= w1) {
          const int64_t at = (int64_t)(2 * wi + (wi == w0 ? 1 : 0)) * (16 * MT) + row;
          st[i] = ws.stats[at];
          x[i] = *reinterpret_cast<const float4*>(ws.part + at * D + d0);
        }
      }
      float m = top;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) m = fmaxf(m, st[i].x);
      const float base = m == -INFINITY ? 0.f : m, keep = __builtin_amdgcn_exp2f(top - base);
      top = m;
      sum *= keep;
      acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const float f = __builtin_amdgcn_exp2f(st[i].x - base);
        sum += f * st[i].y;
        acc.x += f * x[i].x; acc.y += f * x[i].y; acc.z += f * x[i].z; acc.w += f * x[i].w;
      }
    }
    *reinterpret_cast<float4*>(&s_acc[group][d0]) = acc;
    if (d0 == 0) {
      s_top[group] = top;
      s_sum[group] = sum;
    }
    __syncthreads();
  }
  if (group != 0) return;
  if (units > 0) {
#pragma unroll
    for (int x = 1; x < kGroups; ++x) top = fmaxf(top, s_top[x]);
    const float base = top == -INFINITY ? 0.f : top;
    sum = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int x = 0; x < kGroups; ++x) {
      const float4 y = *reinterpret_cast<const float4*>(&s_acc[x][d0]);
      const float f = __builtin_amdgcn_exp2f(s_top[x] - base);
      sum += f * s_sum[x];
      acc.x += f * y.x; acc.y += f * y.y; acc.z += f * y.z; acc.w += f * y.w;
    }
  }
  const int tok = row / a.g, hq = kv * a.g + row - tok * a.g;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<uint2*>(a.out.p + (int64_t)hq * a.out.head + (int64_t)(r.row0 + tok) * a.out.token + d0) =
      make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
  if (a.lse != nullptr && d0 == 0)
    a.lse[(int64_t)hq * a.batch.n_tokens + r.row0 + tok] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// =====================================================================================
// Chunks: many rows per sequence and kv head, bound by the matrix cores.
//
// A workgroup has 128 rows of a (sequence, kv head), 32 for each of its four waves, and goes through the keys that they see in
// tiles of 64, K and V in two LDS buffers each: the next tile is requested while this one is used.  Formulation and tile
// layout are those of the block-sparse kernel: S^T = K Q^T and O^T += V^T P^T with 32x32x16 MFMAs, a row in two lanes, V transposed
// on the way from LDS.  bf16 pages are copied to LDS asynchronously; e4m3 pages pass through registers, where they
// become bf16 once for the four waves (their scales go to the scores and the probabilities in fp32).
// Rows of a kv head's q-heads lie side by side, so the 128 rows are 128 / g tokens and the diagonal costs little.
// P is rounded to bf16 as above; sums and maxima are fp32.  The tiles are pipelined: the scores of the next tile between the
// exponentials of this one, the second product beside the next maxima.  The running sums are scaled again only where a maximum grows by
// more than 2^8, so exponentials are at most 2^8 (fp32 sums and bf16 P hold that as well as 1).
//
// Measured: 2048 tokens behind 30720, 32/8 heads, d = 128, bf16: 975 to 1049 us by the card = 1092 to 1015 TFLOP/s, where a large library product
// reaches 1379 on this card at its power limit; the matrix cores are busy for 57 % of the cycles, without bank conflicts in LDS, and the VALU
// has most of the others (a score costs its exponential, maximum and sum whatever d is: d = 64 reaches 830 TFLOP/s).  e4m3: 1012 us.
// Where the row tiles are few, they are cut into pieces, which chunk_combine_kernel joins: each into the same number of them, or,
// where sequences of different lengths may be long, by chunk_plan_kernel, one workgroup, which counts the keys and deals.
// =====================================================================================
constexpr int kChunkRows = 128, kChunkKeys = 64, kChunkThreads = 256;

// How the row tiles (slots) are cut.  splits > 0: into so many pieces each.  Otherwise what chunk_plan_kernel leaves: of a slot its
// sequence, its first piece, counted over a kv head, and where its parts lie if it has several; the slots that have several.
struct ChunkPlan {
  int32_t* first_piece;    // [slots + 1]
  int32_t* seq;            // [slots]
  int32_t* first_part;     // [slots]
  int32_t* cut;            // [slots]
  int32_t* head;           // tiles of a piece at most, parts of a kv head, slots that are cut
  int32_t slots, splits;
};
// Of a piece its slot, its sequence, which of the slot's pieces it is, and its place among the kv head's parts.
struct ChunkPiece {
  int slot, seq, nth, part;
};
struct ChunkWs {
  float* part;             // [kv heads][parts][part_rows][D] unscaled sums
  float2* stats;           // [kv heads][parts][part_rows]
  ChunkPlan plan;
  int32_t part_rows;       // rows of a row tile at most
};
// Workgroups go round the eight XCDs; those of an XCD get the same kv heads, whose keys then stay in its L2.  Later row tiles,
// which see more keys, first.  Returns the piece of kv head *kv, or -1.
__device__ __forceinline__ int chunk_piece(int b, int h_kv, int pieces, int* kv) {
  int j;
  if (8 % h_kv == 0) {                                    // 8 / h_kv XCDs share a kv head
    const int share = 8 / h_kv, x = b & 7;
    *kv = x / share;
    j = (b >> 3) * share + x % share;
  } else if (h_kv % 8 == 0) {
    const int i = b >> 3;
    if (pieces == 0 || i / pieces >= h_kv / 8) return -1;
    *kv = (b & 7) + 8 * (i / pieces);
    j = i % pieces;
  } else {
    *kv = b % h_kv;
    j = b / h_kv;
  }
  return pieces - 1 - j;                                  // below 0: none
}
inline int64_t chunk_grid(int h_kv, int64_t pieces) {
  const int share = 8 % h_kv == 0 ? 8 / h_kv : 1;
  return (pieces + share - 1) / share * share * h_kv;
}
// The rows of a slot; rows == 0: none, or not this kernel's.
struct ChunkRows {
  SeqRows r;
  int s, row0, rows;       // first row, rows of the sequence
};
__device__ __forceinline__ ChunkRows chunk_rows(const AttnCall& a, int slot, int s) {
  ChunkRows c;
  c.s = s;
  c.r = seq_rows(a.batch, c.s);
  c.row0 = (slot - (int)((((int64_t)c.r.row0 * a.g) >> 7) + c.s)) * kChunkRows;
  const int rows = min(c.r.n, a.batch.each) * a.g;
  c.rows = rows > a.step_rows && c.row0 >= 0 && c.row0 < rows ? rows : 0;
  return c;
}

__device__ __forceinline__ ChunkRows chunk_rows(const AttnCall& a, int slot) { return chunk_rows(a, slot, seq_at(a.batch, slot, a.g, 7, 1)); }
__device__ __forceinline__ ChunkRows uniform(ChunkRows c) {
  return ChunkRows{{uniform(c.r.row0), uniform(c.r.n), uniform(c.r.length)}, uniform(c.s), uniform(c.row0), uniform(c.rows)};
}
__device__ __forceinline__ KeyRange chunk_keys(const AttnCall& a, const ChunkRows& c) {
  if (c.rows == 0) return KeyRange{0, 0, 0};
  const int pos0 = c.r.length - c.r.n, last = min(c.row0 + kChunkRows, c.rows) - 1;
  return key_range<kChunkKeys>(a, pos0 + c.row0 / a.g, pos0 + last / a.g);
}
__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// A piece is at most 5/4 of the share that each of `workers` workgroups would have of all tiles, and four tiles at least.  A row tile
// is cut into equal pieces, each more than half of that, so that the pieces of cut row tiles are fewer than 8/5 of the workers.
// Measured (one of 1024 tokens at 32K beside prompts of 2000, 1000 and 500, 32/8 heads, d = 128; 6 ragged ones up to 32K, 16/4 heads,
// d = 64): 2 shares 827 and 177 us, 3/2 569 and 200, 5/4 570 and 183; cut evenly 813 and 508.
constexpr int kPlanThreads = 1024, kLeastPiece = 4;
template <int D>
__global__ __launch_bounds__(kPlanThreads) void chunk_plan_kernel(AttnCall a, ChunkPlan plan, int workers) {
  __shared__ int s_sum[3][kPlanThreads / 64];
  __shared__ unsigned long long s_total;
  __shared__ int s_blind[kPlanThreads], s_blinds;
  const int t = threadIdx.x, wave = t >> 6;
  if (t == 0) s_total = 0;
  __syncthreads();
  ChunkRows c = {};                                       // of the last slot that was counted
  int tiles = 0;
  unsigned long long mine = 0;
  for (int slot = t; slot < plan.slots; slot += kPlanThreads) {
    c = chunk_rows(a, slot);
    tiles = chunk_keys(a, c).count();
    mine += (unsigned)tiles;
  }
  atomicAdd(&s_total, mine);                              // whole numbers: in any order
  __syncthreads();
  const unsigned long long all = s_total * a.cache.h_kv;
  const unsigned long long share = (5 * all + 4 * workers - 1) / (4 * workers);
  const int most = max(kLeastPiece, (int)min(share, (unsigned long long)kMaxPlaces));
  int carry[3] = {0, 0, 0};                               // pieces, parts, cut slots in front
  for (int base = 0; base < plan.slots; base += kPlanThreads) {
    const int slot = base + t;
    if (plan.slots > kPlanThreads) {
      c = ChunkRows{};
      if (slot < plan.slots) c = chunk_rows(a, slot);
      tiles = chunk_keys(a, c).count();
    }
    const int pieces = ceil_div(tiles, most), cut = pieces > 1 ? 1 : 0;
    const int own[3] = {pieces, cut * pieces, cut};
    int upto[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) upto[i] = wave_scan_inclusive(own[i]);
    __syncthreads();
    if (t == 0) s_blinds = 0;
    if ((t & 63) == 63)
#pragma unroll
      for (int i = 0; i < 3; ++i) s_sum[i][wave] = upto[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      int total = 0;
      for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w == wave) upto[i] += total;
        total += s_sum[i][w];
      }
      upto[i] += carry[i];
      carry[i] += total;
    }
    if (slot < plan.slots) {
      plan.first_piece[slot] = upto[0] - own[0];
      plan.seq[slot] = c.s;
      plan.first_part[slot] = upto[1] - own[1];
      if (cut) plan.cut[upto[2] - 1] = slot;
    }
    // rows that see nothing
    if (c.rows > 0 && tiles == 0) s_blind[atomicAdd(&s_blinds, 1)] = slot;
    __syncthreads();
    for (int i = 0; i < s_blinds; ++i) {
      const ChunkRows b = chunk_rows(a, s_blind[i]);
      const int n = min(b.row0 + kChunkRows, b.rows) - b.row0;
      for (int x = t; x < n * a.cache.h_kv * (D / 8); x += kPlanThreads) {
        const int d0 = x % (D / 8) * 8, row = b.row0 + x / (D / 8) % n, kv = x / (D / 8) / n;
        const int tok = row / a.g, hq = kv * a.g + row - tok * a.g;
        *reinterpret_cast<uint4*>(a.out.p + (int64_t)hq * a.out.head + (int64_t)(b.r.row0 + tok) * a.out.token + d0) = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse != nullptr && d0 == 0) a.lse[(int64_t)hq * a.batch.n_tokens + b.r.row0 + tok] = -INFINITY;
      }
    }
  }
  if (t == 0) {
    plan.first_piece[plan.slots] = carry[0];
    plan.head[0] = most;
    plan.head[1] = carry[1];
    plan.head[2] = carry[2];
  }
}
__device__ __forceinline__ int chunk_pieces(const ChunkPlan& plan) { return plan.splits > 0 ? plan.slots * plan.splits : plan.first_piece[plan.slots]; }
__device__ __forceinline__ int chunk_parts(const ChunkPlan& plan) { return plan.splits > 0 ? plan.slots * plan.splits : plan.head[1]; }
// Pieces of a slot with so many tiles of keys.
__device__ __forceinline__ int chunk_pieces(const ChunkPlan& plan, int tiles) { return plan.splits > 0 ? plan.splits : ceil_div(tiles, plan.head[0]); }
// A planned call's slot of piece j is the last one whose first piece is at most j.  64 places at a time.
__device__ __forceinline__ ChunkPiece piece_at(const AttnCall& a, const ChunkPlan& plan, int j) {
  if (plan.splits > 0) {
    const int slot = j / plan.splits;
    return ChunkPiece{slot, seq_at(a.batch, slot, a.g, 7, 1), j - slot * plan.splits, j};
  }
  const int lane = threadIdx.x & 63;
  int lo = 0, n = plan.slots;                             // in [lo, lo + n), and lo's first piece is at most j
  while (n > 1) {
    const int step = ceil_div(n, 64), at = lo + lane * step;
    const bool low = at < lo + n && plan.first_piece[at] <= j;
    const int last = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(low) | 1ull);
    const int end = lo + n;
    lo += last * step;
    n = min(step, end - lo);
  }
  lo = uniform(lo);
  const int nth = j - plan.first_piece[lo];
  return ChunkPiece{lo, plan.seq[lo], nth, plan.first_part[lo] + nth};
}

template <int D, bool kE4m3>
__global__ __launch_bounds__(kChunkThreads, D == 256 ? 1 : 2) void chunk_kernel(AttnCall a, ChunkWs ws) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KS = D / 16, DT = D / 32, KT = kChunkKeys / 32;
  constexpr int kRow = D * 2, kTileBytes = kChunkKeys * kRow, kSlab = 32 * kRow;
  constexpr int kPieces = D / 32, kHalf = kPieces / 2;    // 16-byte pieces of a thread, of 32 keys
  constexpr int kCpr = D / 8, kRp = kChunkThreads / kCpr; // pieces of a row, rows of a piece of all threads
  constexpr int kWide = kE4m3 ? D / 64 : 0;               // e4m3: 16-byte loads of a thread
  __shared__ __attribute__((aligned(16))) char lds_k[2 * kTileBytes];
  __shared__ __attribute__((aligned(16))) char lds_v[2 * kTileBytes];
  __shared__ int s_special[2][4];
  const int h_kv = a.cache.h_kv;
  const ChunkPlan& plan = ws.plan;
  int kv = 0;
  const int piece = chunk_piece(blockIdx.x, h_kv, chunk_pieces(plan), &kv);
  if (piece < 0) return;
  const ChunkPiece at = piece_at(a, plan, piece);
  const ChunkRows c = uniform(chunk_rows(a, at.slot, at.seq));
  if (c.rows == 0) return;
  const int t = threadIdx.x, lane = t & 63, wave = uniform(t >> 6), l32 = lane & 31, hf = lane >> 5;
  const int pos0 = c.r.length - c.r.n, last_row = min(c.row0 + kChunkRows, c.rows) - 1;
  const int wg_first = pos0 + c.row0 / a.g, wg_last = pos0 + last_row / a.g;
  const KeyRange keys = chunk_keys(a, c);
  const int pieces = chunk_pieces(plan, keys.count());
  const int c0 = (int)((int64_t)keys.count() * at.nth / pieces), c1 = (int)((int64_t)keys.count() * (at.nth + 1) / pieces);

  // this wave's rows
  const int wave_row0 = c.row0 + wave * 32, row = min(wave_row0 + l32, c.rows - 1);
  const bool idle = wave_row0 >= c.rows;
  const int tok = row / a.g, hq = kv * a.g + row - tok * a.g, row_pos = pos0 + tok;
  const int pos_first = pos0 + wave_row0 / a.g, pos_last = pos0 + min(wave_row0 + 31, c.rows - 1) / a.g;
  bf16x8 qf[KS];
  {
    const uint16_t* qp = a.q.p + (int64_t)hq * a.q.head + (int64_t)(c.r.row0 + tok) * a.q.token + hf * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
  }
  if (D > 128) {                                          // read by the MFMAs only: from AGPRs, in place
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+a"(qf[ks]));
  }

  // offsets: this lane's reads inside a slab of 32 rows, its pieces inside 32 keys of a page
  int koff[KS], voff[D > 128 ? 4 : DT];
  constexpr int kGroups = D > 128 ? 4 : DT;
#pragma unroll
  for (int st = 0; st < KS; ++st) koff[st] = l32 * kRow + (((2 * st + hf) ^ k_row_swizzle<D>(l32)) << 4);
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const int key = 4 * hf + ((lane >> 2) & 3);
    voff[i] = key * kRow + ((i ^ v_row_swizzle<D>(key)) << 6) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  }
  int k_lane[2], v_lane[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = i * kRp + t / kCpr;
    k_lane[i] = r * kRow + (((t % kCpr) ^ k_row_swizzle<D>(r)) << 4);
    v_lane[i] = r * kRow + (((t % kCpr) ^ (v_row_swizzle<D>(r) << 2)) << 4);
  }

  // ---- tiles: entries of the page table held 64 a time, one a lane, as addresses of the head's K (0: no page), with scales ----
  const int32_t* table = a.batch.table + (int64_t)c.s * a.batch.max_pages;
  constexpr int kPageRow = kE4m3 ? D : kRow;
  const char* k_head = a.cache.k + (int64_t)kv * a.cache.page * kPageRow;
  const int64_t v_from_k = a.cache.v - a.cache.k;
  int held_from = -64;
  uint32_t held_lo = 0, held_hi = 0;
  float held_ks = 0.f, held_vs = 0.f;
  auto lane_value = [](uint32_t x, int lane) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); };
  // e4m3: the values' scale is a power of two, which the conversion to bf16 applies, times vs in [1, 2): 1 for scales of
  // prism_cache_append, and the probabilities need no factor.
  struct Half {
    uint64_t k;                                           // address of its K; V lies v_from_k behind
    int bytes;                                            // that are there: what lies behind reads as zero; 0: no page
    float ks, vs, v_power;
  };
  struct Tile {
    int first;                                            // its first key
    Half half[2];
  };
  auto locate = [&](int list_at) __attribute__((always_inline)) {
    Tile x;
    x.first = keys.tile(list_at) * kChunkKeys;
#pragma unroll
    for (int hv = 0; hv < 2; ++hv) {
      const int tk = x.first + 32 * hv, e = tk >> a.cache.page_shift;
      if ((unsigned)(e - held_from) >= 64u) {
        held_from = e;
        const int mine = e + lane;
        const int id = mine < a.batch.max_pages ? table[mine] : -1;
        const bool there = id >= 0 && id < a.cache.n_pages;
        const uint64_t at = there ? (uint64_t)k_head + (uint64_t)id * a.cache.page_stride : 0;
        held_lo = (uint32_t)at;
        held_hi = (uint32_t)(at >> 32);
        if (kE4m3) {
          const int64_t sc = (int64_t)(there ? id : 0) * h_kv + kv;
          held_ks = a.cache.k_scale[sc];
          held_vs = a.cache.v_scale[sc];
        }
      }
      Half& y = x.half[hv];
      const int l = e - held_from;
      const uint64_t at = (uint64_t)lane_value(held_hi, l) << 32 | lane_value(held_lo, l);
      y.k = at + (tk & (a.cache.page - 1)) * kPageRow;
      const int there = c.r.length - tk;
      y.bytes = at == 0 || there <= 0 ? 0 : (there >= 32 ? 32 : there) * kPageRow;
      if (kE4m3) {
        y.ks = __uint_as_float(lane_value(__float_as_uint(held_ks), l));
        const uint32_t vs = lane_value(__float_as_uint(held_vs), l);
        y.vs = __uint_as_float((vs & 0x007FFFFFu) | 0x3F800000u);
        y.v_power = __uint_as_float(vs & 0x7F800000u);
      }
    }
    return x;
  };
  const int wave_base = uniform(t & ~63);
  // piece i of K or V of a tile (its halves' resources), to buffer b
  auto resources = [&](TileRsrc(&rs)[2], const Tile& x, int64_t from_k) __attribute__((always_inline)) {
#pragma unroll
    for (int hv = 0; hv < 2; ++hv) rs[hv] = make_tile_rsrc((const void*)(x.half[hv].k + from_k), x.half[hv].bytes);
  };
  auto copy_k = [&](const TileRsrc(&rs)[2], int i, int b) __attribute__((always_inline)) {
    const int j = i % kHalf;
    async_piece(rs[i / kHalf], k_lane[j & 1], (j & 2) * kRp * kRow, (uint32_t)(size_t)lds_k + b * kTileBytes + (i * kChunkThreads + wave_base) * 16);
  };
  auto copy_v = [&](const TileRsrc(&rs)[2], int i, int b) __attribute__((always_inline)) {
    const int j = i % kHalf;
    async_piece(rs[i / kHalf], v_lane[j & 1], (j & 2) * kRp * kRow, (uint32_t)(size_t)lds_v + b * kTileBytes + (i * kChunkThreads + wave_base) * 16);
  };
  // e4m3: 16 values a piece, through registers
  u32x4 kx[kWide > 0 ? kWide : 1], vx[kWide > 0 ? kWide : 1];
  constexpr int kWideCpr = D / 16, kWideRp = kChunkThreads / kWideCpr;    // rows of a piece of all threads: 64, 32, 16
  auto wide_half = [&](int i) __attribute__((always_inline)) { return kWideRp == 64 ? uniform(t / kWideCpr >> 5) : i * kWideRp / 32; };
  auto request = [&](u32x4(&to)[kWide > 0 ? kWide : 1], const Tile& x, int64_t from_k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kWide; ++i) {
      const int r = i * kWideRp + t / kWideCpr, hv = wide_half(i);
      to[i] = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc((const void*)((hv ? x.half[1].k : x.half[0].k) + from_k), hv ? x.half[1].bytes : x.half[0].bytes),
                                                    (r & 31) * D + (t % kWideCpr) * 16, 0, 0);
    }
  };
  auto deliver_k = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kWide; ++i) {
      const int r = i * kWideRp + t / kWideCpr, ch = 2 * (t % kWideCpr);
#pragma unroll
      for (int hv = 0; hv < 2; ++hv)
        *reinterpret_cast<u32x4*>(lds_k + b * kTileBytes + r * kRow + (((ch + hv) ^ k_row_swizzle<D>(r)) << 4)) = bf16_of_e4m3(kx[i][2 * hv], kx[i][2 * hv + 1], 1.f);
    }
  };
  auto deliver_v = [&](int b, const Tile& x) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kWide; ++i) {
      const int r = i * kWideRp + t / kWideCpr, ch = 2 * (t % kWideCpr);
      const float power = wide_half(i) ? x.half[1].v_power : x.half[0].v_power;
#pragma unroll
      for (int hv = 0; hv < 2; ++hv)
        *reinterpret_cast<u32x4*>(lds_v + b * kTileBytes + r * kRow + (((ch + hv) ^ (v_row_swizzle<D>(r) << 2)) << 4)) = bf16_of_e4m3(vx[i][2 * hv], vx[i][2 * hv + 1], power);
    }
  };
  // A operand of O^T: dims 32*dt .. +31, keys 16*st + 8*(j/4) + 4*hf + j%4
  auto v_frag = [&](int dt, int st, int b) __attribute__((always_inline)) {
    typedef __attribute__((address_space(3))) bf16x4* lv4_t;
    const char* p = lds_v + b * kTileBytes + voff[dt % kGroups] + (dt / kGroups) * (kGroups * 64) + st * (16 * kRow);
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lv4_t)p), y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lv4_t)(p + 8 * kRow));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const int window = a.window > 0 ? a.window : 0x40000000;
  constexpr int kDepth = 3;                               // LDS reads ahead of their MFMA
  const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

  // S^T of a tile whose K is in buffer kBuf, with `between(i)` behind MFMA i
  auto scores = [&](f32x16(&sc)[KT], auto buf_tag, auto between) __attribute__((always_inline)) {
    constexpr int kBuf = decltype(buf_tag)::value, kSteps = KT * KS;
    static_assert(kSteps >= kDepth, "pipeline deeper than the phase");
    const char* kb = lds_k + kBuf * kTileBytes;
    bf16x8 fr[kDepth];
#pragma unroll
    for (int i = 0; i < kDepth; ++i) fr[i] = *reinterpret_cast<const bf16x8*>(kb + (i % KT) * kSlab + koff[i / KT]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int kt = i % KT, ks = i / KT, j = i + kDepth;
      sc[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % kDepth], qf[ks], ks == 0 ? zero16 : sc[kt], 0, 0, 0);
      if (j < kSteps) fr[i % kDepth] = *reinterpret_cast<const bf16x8*>(kb + (j % KT) * kSlab + koff[j / KT]);
      between(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // whether all rows of the workgroup see all of a tile
  auto inside = [&](const Tile& x) __attribute__((always_inline)) {
    return (x.half[0].bytes != 0) & (x.half[1].bytes != 0) & (x.first + kChunkKeys - 1 <= wg_first) &
           ((x.first > wg_last - window) | (x.first + kChunkKeys - 1 < a.sinks));
  };
  // scores of keys that a row does not see (without branches, as in step_kernel)
  auto hide = [&](f32x16(&sc)[KT], const Tile& x) __attribute__((always_inline)) {
    int pos = row_pos;
    asm volatile("" : "+v"(pos));                         // formed here, not kept from in front of the loop
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = x.first + kt * 32 + 8 * (r >> 2) + 4 * hf + (r & 3);
        const bool s = (x.half[kt].bytes != 0) & (key <= pos) & ((key > pos - window) | (key < a.sinks));
        sc[kt][r] = s ? sc[kt][r] : -INFINITY;
      }
  };
  // The reference of the exponentials (mx: this lane's maximum of each 32 keys).  It follows the maximum only when that is more than
  // 2^8 ahead, so that the sums are seldom rescaled: p stays below 2^8, whose rounding to bf16 is as good, and the sums
  // are far from the end of fp32.
  auto raise = [&](const float (&mx)[KT], const Tile& x) __attribute__((always_inline)) {
    float y = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) y = fmaxf(y, mx[kt] * (kE4m3 ? a.scale * x.half[kt].ks : a.scale));
    y = other_half_max(y);
    if (__builtin_amdgcn_ballot_w64(y > m_run + 8.f) != 0) {        // some row is that far ahead
      const float m_new = fmaxf(m_run, y);
      const float keep = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= keep;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= keep;
      m_run = m_new;
    }
  };

  bool specials = false;
  Tile now = {}, next = {}, after = {};
  f32x16 sa[KT], sb[KT];                                  // scores of this tile and of the next one, by turns
  // Tile `now`, its scores in sc_now and below m_run; K of `next` and V of `now` are in LDS.
  //   phase 1: S^T of the next tile, between its MFMAs the exponentials of this one and the requests of K two tiles and V one
  //            tile ahead
  //   phase 2: O^T += V^T P^T of this tile, between its MFMAs the maximum of the next one's scores
  // A MFMA leaves its wave room for about five vector instructions; with scores, softmax and product one after the other the two
  // waves of a SIMD did not fill each other's gaps (MFMAs and vector instructions together were 94 % of the time).
  auto step = [&](auto buf_tag, auto last_tag, f32x16(&sc_now)[KT], f32x16(&sc_next)[KT], int list_at) __attribute__((always_inline)) {
    constexpr int kBuf = decltype(buf_tag)::value;        // V of `now`, K of the tile two ahead
    constexpr bool kLast = decltype(last_tag)::value;     // no next tile
    const bool two = list_at + 2 < c1;
    TileRsrc krs[2], vrs[2];
    if (!kLast) {
      if (two) after = locate(list_at + 2);
      if (kE4m3) {
        request(vx, next, v_from_k);
        if (two) request(kx, after, 0);
      } else {
        resources(vrs, next, v_from_k);
        resources(krs, after, 0);
      }
    }
    const float base = m_run == -INFINITY ? 0.f : m_run;  // nothing seen yet: all p are 0
    float by[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) by[kt] = kE4m3 ? a.scale * now.half[kt].ks : a.scale;
    u32x4 pf[KT][2];
    float sum0 = 0.f, sum1 = 0.f;
    auto phase1 = [&](auto scaled) __attribute__((always_inline)) {
      auto pair = [&](int e) __attribute__((always_inline)) {       // scores 2e, 2e + 1 of this lane
        const int kt = e >> 3, r = 2 * (e & 7);
        float p0 = __builtin_amdgcn_exp2f(fmaf(sc_now[kt][r], by[kt], -base));
        float p1 = __builtin_amdgcn_exp2f(fmaf(sc_now[kt][r + 1], by[kt], -base));
        sum0 += p0;
        sum1 += p1;
        if (decltype(scaled)::value) {
          p0 *= now.half[kt].vs;
          p1 *= now.half[kt].vs;
        }
        uint32_t w = bf16_pair(p0, p1);
        asm volatile("" : "+v"(w), "+v"(sum0), "+v"(sum1));         // here, not where the compiler first needs it
        pf[kt][r >> 3][(r & 7) >> 1] = w;
      };
      constexpr int kPairs = 8 * KT;
      if constexpr (kLast) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) pair(e);
      } else {
        constexpr int kSteps = KT * KS, kEvery = kSteps / (2 * kPieces);
        static_assert(kSteps % (2 * kPieces) == 0, "pieces between the MFMAs");
        scores(sc_next, std::integral_constant<int, 1 - kBuf>{}, [&](int i) __attribute__((always_inline)) {
          if (!kE4m3 && i % kEvery == 0) {
            const int p = i / kEvery;
            if (p < kPieces) copy_v(vrs, p, 1 - kBuf);
            else if (two) copy_k(krs, p - kPieces, kBuf);
          }
#pragma unroll
          for (int e = i * kPairs / kSteps; e < (i + 1) * kPairs / kSteps; ++e) pair(e);
        });
      }
    };
    __builtin_amdgcn_s_setprio(1);
    if (kE4m3 && (now.half[0].vs != 1.f || now.half[1].vs != 1.f))
      phase1(std::true_type{});
    else
      phase1(std::false_type{});
    __builtin_amdgcn_s_setprio(0);
    l_run += sum0 + sum1;

    if (!kLast && !inside(next)) hide(sc_next, next);
    // 0 * NaN is NaN: in a tile that not every row of the workgroup sees all of, infinities and NaN among the values leave
    // before the product; the rows that see them get them at the end
    if (!inside(now)) {
      constexpr int kQuarter = kTileBytes / 4;
      char* vb = lds_v + kBuf * kTileBytes;
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < kQuarter / 1024; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(vb + wave * kQuarter + i * 1024 + lane * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= special_bits<false>(w[e]);
      }
      const bool some = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
      if (lane == 0) s_special[kBuf][wave] = some;
      tile_barrier();
      const int special = uniform(s_special[kBuf][0] | s_special[kBuf][1] | s_special[kBuf][2] | s_special[kBuf][3]);
      if (special != 0) {
        specials = true;
#pragma unroll 1
        for (int i = 0; i < kQuarter / 1024; ++i) {
          u32x4* w = reinterpret_cast<u32x4*>(vb + wave * kQuarter + i * 1024 + lane * 16);
          *w = u32x4{without_specials<false>((*w)[0]), without_specials<false>((*w)[1]), without_specials<false>((*w)[2]), without_specials<false>((*w)[3])};
        }
        tile_barrier();
      }
    }

    __builtin_amdgcn_s_setprio(1);
    float mx[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) mx[kt] = -INFINITY;
    {
      constexpr int kSteps = DT * KT * 2, kScores = 16 * KT;
      static_assert(kSteps >= kDepth, "pipeline deeper than the phase");
      bf16x8 fr[kDepth];
#pragma unroll
      for (int i = 0; i < kDepth; ++i) fr[i] = v_frag(i % DT, i / DT, kBuf);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int dt = i % DT, st = i / DT;
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % kDepth], __builtin_bit_cast(bf16x8, pf[st >> 1][st & 1]), o[dt], 0, 0, 0);
        if (i + kDepth < kSteps) fr[i % kDepth] = v_frag((i + kDepth) % DT, (i + kDepth) / DT, kBuf);
        if (!kLast) {
#pragma unroll
          for (int e = i * kScores / kSteps; e < (i + 1) * kScores / kSteps; ++e) mx[e >> 4] = fmaxf(mx[e >> 4], sc_next[e >> 4][e & 15]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if (!kLast) {
      raise(mx, next);
      if (kE4m3) {
        deliver_v(1 - kBuf, next);
        if (two) deliver_k(kBuf);
      }
      wait_async_loads();                                 // this wave's share of the tiles ahead has landed
      tile_barrier();                                     // ... everyone's, and everyone is done with this tile
      now = next;
      next = after;
    }
  };

  if (c0 < c1) {
    // K and V of the first tile, K of the second
    now = locate(c0);
    if (c0 + 1 < c1) next = locate(c0 + 1);
    if (kE4m3) {
      request(kx, now, 0);
      request(vx, now, v_from_k);
      deliver_k(0);
      deliver_v(0, now);
      if (c0 + 1 < c1) {
        request(kx, next, 0);
        deliver_k(1);
      }
    } else {
      TileRsrc krs[2], vrs[2];
      resources(krs, now, 0);
      resources(vrs, now, v_from_k);
#pragma unroll
      for (int i = 0; i < kPieces; ++i) copy_k(krs, i, 0);
#pragma unroll
      for (int i = 0; i < kPieces; ++i) copy_v(vrs, i, 0);
      if (c0 + 1 < c1) {
        resources(krs, next, 0);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) copy_k(krs, i, 1);
      }
    }
    wait_async_loads();
    tile_barrier();
    scores(sa, std::integral_constant<int, 0>{}, [](int) {});
    if (!inside(now)) hide(sa, now);
    {
      float mx[KT];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        mx[kt] = sa[kt][0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx[kt] = fmaxf(mx[kt], sa[kt][r]);
      }
      raise(mx, now);
    }
    tile_barrier();                                       // everyone is done with K of the first tile
    int i = c0;
    for (; i + 2 < c1; i += 2) {
      step(std::integral_constant<int, 0>{}, std::false_type{}, sa, sb, i);
      step(std::integral_constant<int, 1>{}, std::false_type{}, sb, sa, i + 1);
    }
    if (i + 1 < c1) {
      step(std::integral_constant<int, 0>{}, std::false_type{}, sa, sb, i);
      step(std::integral_constant<int, 1>{}, std::true_type{}, sb, sa, i + 1);
    } else {
      step(std::integral_constant<int, 0>{}, std::true_type{}, sa, sb, i);
    }
  }

  if (specials) {                                         // rare: the tiles once more; p > 0 times an infinity or NaN is that
#pragma unroll 1
    for (int i = c0; i < c1; ++i) {
      const Tile x = locate(i);
      if (inside(x)) continue;
#pragma unroll 1
      for (int j = 0; j < kChunkKeys; ++j) {
        constexpr int kElem = kE4m3 ? 1 : 2;
        const Half& y = j < 32 ? x.half[0] : x.half[1];
        const int key = x.first + j;
        const bool s = (y.bytes != 0) & (key <= row_pos) & ((key > row_pos - window) | (key < a.sinks));
        if (!s) continue;
        const char* vr = (const char*)(y.k + v_from_k) + (j & 31) * (D * kElem);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const char* at = vr + (dt * 32 + 8 * (r >> 2) + 4 * hf + (r & 3)) * kElem;
            float z;
            if constexpr (kE4m3)
              z = __builtin_amdgcn_cvt_f32_fp8(*reinterpret_cast<const uint8_t*>(at), 0);
            else
              z = bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(at));
            o[dt][r] += fabsf(z) < INFINITY ? 0.f : z;
          }
      }
    }
  }
  const float l = other_half_sum(l_run);
  if (wave_row0 + l32 >= c.rows) return;
  if (pieces == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* op = a.out.p + (int64_t)hq * a.out.head + (int64_t)(c.r.row0 + tok) * a.out.token;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<uint2*>(op + dt * 32 + q * 8 + hf * 4) =
            make_uint2(bf16_pair(o[dt][4 * q] * inv, o[dt][4 * q + 1] * inv), bf16_pair(o[dt][4 * q + 2] * inv, o[dt][4 * q + 3] * inv));
    if (a.lse != nullptr && hf == 0)
      a.lse[(int64_t)hq * a.batch.n_tokens + c.r.row0 + tok] = l == 0.f ? -INFINITY : (m_run + log2f(l)) * kLn2;
  } else {
    const int64_t place = ((int64_t)kv * chunk_parts(plan) + at.part) * ws.part_rows + wave * 32 + l32;
    float* pp = ws.part + place * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(pp + dt * 32 + q * 8 + hf * 4) = make_float4(o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]);
    if (hf == 0) ws.stats[place] = make_float2(m_run, l);
  }
#endif
}

// Joins the parts of the rows of cut row tiles.  The groups of D / 4 threads of a workgroup have a row each, or (kOneRow, for calls of
// few row tiles, which have many parts) every so many parts of one row, each with a maximum of its own.
template <int D, bool kOneRow>
__global__ __launch_bounds__(kChunkThreads) void chunk_combine_kernel(AttnCall a, ChunkWs ws) {
  constexpr int kGroups = kChunkThreads * 4 / D, kAtOnce = 4;
  __shared__ float s_acc[kGroups][D];
  __shared__ float s_top[kGroups], s_sum[kGroups];
  const ChunkPlan& plan = ws.plan;
  int slot = blockIdx.x, seq = 0, part = slot * plan.splits;
  const int kv = blockIdx.y;
  if (plan.splits > 0) {
    seq = seq_at(a.batch, slot, a.g, 7, 1);
  } else {
    if (slot >= plan.head[2]) return;
    slot = plan.cut[slot];
    seq = plan.seq[slot];
    part = plan.first_part[slot];
  }
  const ChunkRows c = uniform(chunk_rows(a, slot, seq));
  if (c.rows == 0) return;
  const int group = threadIdx.x / (D / 4), d0 = threadIdx.x % (D / 4) * 4;
  const int x = kOneRow ? blockIdx.z : blockIdx.z * kGroups + group, row = c.row0 + x;
  if (kOneRow && row >= c.rows) return;
  const int parts = chunk_pieces(plan, chunk_keys(a, c).count());
  const int64_t place = ((int64_t)kv * chunk_parts(plan) + part) * ws.part_rows + x;
  float top = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int w = kOneRow ? group : 0; w < parts && row < c.rows; w += kAtOnce * (kOneRow ? kGroups : 1)) {
    float2 st[kAtOnce];
    float4 y[kAtOnce];
    float m = top;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int wi = w + i * (kOneRow ? kGroups : 1);
      st[i] = make_float2(-INFINITY, 0.f);
      y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (wi < parts) {
        st[i] = ws.stats[place + (int64_t)wi * ws.part_rows];
        y[i] = *reinterpret_cast<const float4*>(ws.part + (place + (int64_t)wi * ws.part_rows) * D + d0);
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) m = fmaxf(m, st[i].x);
    const float base = m == -INFINITY ? 0.f : m, keep = __builtin_amdgcn_exp2f(top - base);
    top = m;
    sum *= keep;
    acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float f = __builtin_amdgcn_exp2f(st[i].x - base);
      sum += f * st[i].y;
      acc.x += f * y[i].x; acc.y += f * y[i].y; acc.z += f * y[i].z; acc.w += f * y[i].w;
    }
  }
  if constexpr (kOneRow) {
    *reinterpret_cast<float4*>(&s_acc[group][d0]) = acc;
    if (d0 == 0) {
      s_top[group] = top;
      s_sum[group] = sum;
    }
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int i = 1; i < kGroups; ++i) top = fmaxf(top, s_top[i]);
    const float base = top == -INFINITY ? 0.f : top;
    sum = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const float4 y = *reinterpret_cast<const float4*>(&s_acc[i][d0]);
      const float f = __builtin_amdgcn_exp2f(s_top[i] - base);
      sum += f * s_sum[i];
      acc.x += f * y.x; acc.y += f * y.y; acc.z += f * y.z; acc.w += f * y.w;
    }
  } else if (row >= c.rows) {
    return;
  }
  const int tok = row / a.g, hq = kv * a.g + row - tok * a.g;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<uint2*>(a.out.p + (int64_t)hq * a.out.head + (int64_t)(c.r.row0 + tok) * a.out.token + d0) =
      make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
  if (a.lse != nullptr && d0 == 0)
    a.lse[(int64_t)hq * a.batch.n_tokens + c.r.row0 + tok] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// =====================================================================================
// Dispatch
// =====================================================================================
constexpr int kWorkers = 512;                             // two workgroups a CU

struct AttnPlan {
  int step_rows;           // see AttnCall
  int mt, workers, rows;   // steps: 16-row tiles, workgroups (0: none of the call's sequences is one), rows of a kv head at most
  int slots, splits;       // chunks: row tiles of a kv head (0: none), parts of each (0: planned on the device)
  int chunk_workers, parts, part_rows;           // workgroups that fill the chip; parts in all and rows of a part, at most
  size_t part_bytes, chunk_part_bytes, chunk_stats_bytes, steps_bytes, bytes;
};
// Which kernels a call needs.  Up to 32 rows (16 at d = 256, where two row tiles do not fit the registers) a sequence and kv
// head is a step's: us as a step / as a chunk, 64 sequences of 4096, 28 rows, d = 64 56 / 80 (e4m3 47 / 100), d = 128 107 / 114 (e4m3
// 61 / 127); 16 of 8192, 16 rows, d = 256 190 / 192 (e4m3 103 / 174).  The lengths of a ragged batch are on the device: if its longest
// sequence has more rows, all are a chunk's, single tokens in row tiles of their own beside the others, as long as the sequences
// are short (below) and do not fill the chip by themselves; otherwise both kernels are launched, and each leaves the
// other's sequences; steps are then those of one row tile.  us with one / both kernels, a chunk of 512 tokens and single ones of others: 7 of
// 1024 (window), 32/8 heads, d = 128 35 / 46 (e4m3 39 / 48), 63 of them 87 / 90 (87 / 76); 7 of 8100 119 / 138 (132 / 136); 7 of 16000
// 259 / 238 (283 / 200), 31 of them 551 / 486 (437 / 339).
//
// Row tiles of chunks are cut where they are fewer than the workgroups that fill the chip, into parts of four tiles of keys at
// least.  The host counts them only, which is right for one sequence and for short ones.  Where a row tile may have 128 tiles of
// keys (8192 keys, 40 us on its own) and there are several sequences, they are planned: 64 sequences of 5 tokens behind 30 to 32000,
// d = 64, 527 -> 110 us; 4 of 40 behind 16384, 88 -> 91.  Planned always, 4 of 512 with a window of 4096 went 142 -> 150 us
// and the ragged chunks of a windowed e4m3 batch 50 -> 56: the plan and the second look at it are two launches more.
constexpr int kPlannedTiles = 128;
static AttnPlan plan_of(const prism_cache* c, const prism_batch* b, int n_q_heads, int window, int sinks) {
  AttnPlan p = {};
  const int g = n_q_heads / c->n_kv_heads;
  const int64_t rows = (int64_t)b->max_tokens * g;
  p.bytes = 256;
  if (b->n_seqs == 0 || b->n_tokens == 0) return p;
  const bool steps_only = rows <= (c->head_dim == 256 ? 16 : 32);
  const bool ragged = b->cu_tokens != nullptr && b->n_seqs > 1;
  const int64_t all = (int64_t)b->max_pages * c->page, band = (int64_t)window + sinks + kChunkRows;
  const int64_t keys = window > 0 && band < all ? band : all;
  const bool planned = b->n_seqs > 1 && keys >= kPlannedTiles * kChunkKeys;
  p.chunk_workers = c->head_dim == 256 ? kWorkers / 2 : kWorkers;
  if (steps_only || (ragged && g <= 16 && (planned || (int64_t)b->n_seqs * c->n_kv_heads >= p.chunk_workers))) {
    p.mt = steps_only && rows > 16 ? 2 : 1;
    p.step_rows = 16 * p.mt;
    p.rows = (int)(rows < p.step_rows ? rows : p.step_rows);
    const int64_t units = (int64_t)b->n_seqs * c->n_kv_heads * (((int64_t)b->max_pages * c->page + 127) / 128);
    // One workgroup a CU where two do not fit the registers without spilling: d = 256, and two row tiles of bf16.  us with one / two,
    // 16 sequences of 8192, 32 rows: d = 128 bf16 106 / 132, e4m3 69 / 58; d = 64 bf16 55 / 57, e4m3 55 / 43.  d = 256, 4 rows: bf16 101 / 220,
    // e4m3 50 / 53.
    const int most = c->head_dim == 256 || (p.mt > 1 && c->dtype == PRISM_CACHE_BF16) ? kWorkers / 2 : kWorkers;
    p.workers = units < most ? (int)units : most;
    const size_t slots = 2 * (size_t)p.workers * 16 * p.mt;
    p.part_bytes = align_up(slots * c->head_dim * sizeof(float), 256);
    p.steps_bytes = p.part_bytes + align_up(slots * sizeof(float2), 256);
  }
  if (!steps_only) {
    p.slots = (int)(((int64_t)b->n_tokens * g) >> 7) + b->n_seqs;
    p.part_rows = rows < kChunkRows ? (int)rows : kChunkRows;
    const int64_t row_tiles = (int64_t)p.slots * c->n_kv_heads;
    if (!planned) {
      const int64_t n = p.chunk_workers / row_tiles, most = (keys + 4 * kChunkKeys - 1) / (4 * kChunkKeys);
      p.splits = n <= 1 || most <= 1 ? 1 : (int)(n < most ? n : most);
      p.parts = p.splits > 1 ? (int)row_tiles * p.splits : 0;
    } else {
      p.parts = (8 * p.chunk_workers + 4) / 5;                      // see chunk_plan_kernel
    }
    const size_t part_rows = (size_t)p.parts * p.part_rows;
    p.chunk_part_bytes = align_up(part_rows * c->head_dim * sizeof(float), 256);
    p.chunk_stats_bytes = align_up(part_rows * sizeof(float2), 256);
    p.bytes = 256 + p.chunk_part_bytes + p.chunk_stats_bytes + (p.splits > 0 ? 0 : align_up((4 * (size_t)p.slots + 4) * sizeof(int32_t), 256));
  }
  p.bytes += p.steps_bytes;
  return p;
}

static int check_attn(const prism_cache* cache, const prism_batch* batch, int n_q_heads) {
  int rc = check_cache(cache);
  if (rc != PRISM_OK || (rc = check_batch(cache, batch)) != PRISM_OK) return rc;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0) return PRISM_ERR_INVALID_ARG;
  if (n_q_heads > kMaxHeads) return PRISM_ERR_UNSUPPORTED;
  if ((int64_t)batch->n_tokens * n_q_heads > kMaxRows || (int64_t)batch->n_seqs * cache->n_kv_heads > kMaxSeqHeads) return PRISM_ERR_UNSUPPORTED;
  return PRISM_OK;
}

template <int D, bool kE4m3, int MT>
static int launch_steps(const AttnCall& a, const AttnPlan& p, char* ws, hipStream_t st) {
  const StepWs w = {reinterpret_cast<float*>(ws), reinterpret_cast<float2*>(ws + p.part_bytes)};
  hipLaunchKernelGGL((step_kernel<D, kE4m3, MT>), dim3(p.workers), dim3(kStepThreads), 0, st, a, w);
  hipLaunchKernelGGL((combine_kernel<D, MT>), dim3(a.batch.n_seqs, a.cache.h_kv, p.rows), dim3(kStepThreads), 0, st, a, w, p.workers);
  return launch_status();
}
template <int D, bool kE4m3>
static int launch_attn(const AttnCall& a, const AttnPlan& p, char* ws, hipStream_t st) {
  if (p.workers > 0) {
    int rc = PRISM_OK;
    if constexpr (D < 256) {
      rc = p.mt == 2 ? launch_steps<D, kE4m3, 2>(a, p, ws, st) : launch_steps<D, kE4m3, 1>(a, p, ws, st);
    } else {
      rc = launch_steps<D, kE4m3, 1>(a, p, ws, st);
    }
    if (rc != PRISM_OK || p.slots == 0) return rc;
  }
  char* cw = ws + p.steps_bytes;
  int32_t* lists = reinterpret_cast<int32_t*>(cw + p.chunk_part_bytes + p.chunk_stats_bytes);
  const size_t n = p.slots;
  const ChunkPlan plan = {lists, lists + n + 1, lists + 2 * n + 1, lists + 3 * n + 1, lists + 4 * n + 1, p.slots, p.splits};
  const ChunkWs w = {reinterpret_cast<float*>(cw), reinterpret_cast<float2*>(cw + p.chunk_part_bytes), plan, p.part_rows};
  const int h_kv = a.cache.h_kv;
  int64_t pieces = n * p.splits, joined = p.splits > 1 ? p.slots : 0;
  if (p.splits == 0) {
    hipLaunchKernelGGL((chunk_plan_kernel<D>), dim3(1), dim3(kPlanThreads), 0, st, a, plan, p.chunk_workers);
    pieces = n + p.parts / h_kv + 1;
    joined = p.parts / 2 / h_kv + 1 < p.slots ? p.parts / 2 / h_kv + 1 : p.slots;
  }
  hipLaunchKernelGGL((chunk_kernel<D, kE4m3>), dim3((unsigned)chunk_grid(h_kv, pieces)), dim3(kChunkThreads), 0, st, a, w);
  if (joined == 0) return launch_status();
  if ((int64_t)p.slots * h_kv <= 32)
    hipLaunchKernelGGL((chunk_combine_kernel<D, true>), dim3((unsigned)joined, h_kv, p.part_rows), dim3(kChunkThreads), 0, st, a, w);
  else
    hipLaunchKernelGGL((chunk_combine_kernel<D, false>), dim3((unsigned)joined, h_kv, (p.part_rows * D + kChunkThreads * 4 - 1) / (kChunkThreads * 4)),
                       dim3(kChunkThreads), 0, st, a, w);
  return launch_status();
}
template <int D>
static int launch_for(bool e4m3, const AttnCall& a, const AttnPlan& p, char* ws, hipStream_t st) {
  return e4m3 ? launch_attn<D, true>(a, p, ws, st) : launch_attn<D, false>(a, p, ws, st);
}

}  // namespace prism

using namespace prism;

extern "C" int prism_cache_attn_workspace_bytes(const prism_cache* cache, const prism_batch* batch, int n_q_heads, size_t* bytes) {
  const int rc = check_attn(cache, batch, n_q_heads);
  if (rc != PRISM_OK) return rc;
  if (bytes == nullptr) return PRISM_ERR_INVALID_ARG;
  *bytes = plan_of(cache, batch, n_q_heads, 0, 0).bytes;        // a window takes away keys, and with them parts, or the plan
  return PRISM_OK;
}

extern "C" int prism_cache_attn(const prism_cache* cache, const prism_batch* batch, const prism_cache_attn_params* params,
                                const prism_rows* q, const prism_rows* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (params == nullptr) return PRISM_ERR_INVALID_ARG;
  int rc = check_attn(cache, batch, params->n_q_heads);
  if (rc != PRISM_OK) return rc;
  if (params->window < 0 || params->sinks < 0 || !(params->scale >= 0.f) || !(params->scale < INFINITY)) return PRISM_ERR_INVALID_ARG;
  const int d = cache->head_dim, T = batch->n_tokens, h = params->n_q_heads;
  if (T == 0) return PRISM_OK;
  if ((rc = check_cache_memory(cache)) != PRISM_OK || (rc = check_rows(q, h, T, d, false)) != PRISM_OK ||
      (rc = check_rows(out, h, T, d, true)) != PRISM_OK || (rc = check_in_place(q, out, h, T)) != PRISM_OK)
    return rc;
  // positions lie between -2^27 and 2^30: a window that is longer sees as much, and position - window stays in 32 bits
  const int window = params->window < 1 << 30 ? params->window : 1 << 30;
  const AttnPlan plan = plan_of(cache, batch, h, window, params->sinks);
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < plan.bytes) return PRISM_ERR_WORKSPACE;
  const float scale = params->scale > 0.f ? params->scale : 1.f / sqrtf((float)d);
  const AttnCall a = {rows_of(q), rows_of(out), lse, cache_view(cache), batch_view(batch), h, h / cache->n_kv_heads,
                      window, params->sinks, scale * kLog2e, plan.step_rows};
  const bool e4m3 = cache->dtype == PRISM_CACHE_E4M3;
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (d) {
    case 64: return launch_for<64>(e4m3, a, plan, ws, st);
    case 128: return launch_for<128>(e4m3, a, plan, ws, st);
    default: return launch_for<256>(e4m3, a, plan, ws, st);
  }
}
