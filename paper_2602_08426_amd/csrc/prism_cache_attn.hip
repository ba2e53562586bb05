// Attention of new tokens over the paged cache (gfx950): prism_cache_attn.
//
// The rows of a (sequence, kv head) are its new tokens times the q-heads of the kv head: row r = token r / g, head r % g,
// so that a tile of keys and values is read once for all of them.
#include "prism_cache.h"

namespace prism {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const char* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, bytes, 0x00020000);
}
// a value that is the same in all lanes, in a scalar register
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// What the kernels need to know of a call.
struct AttnCall {
  Rows q, out;
  float* lse;
  CacheView cache;
  BatchView batch;         // each = max_tokens
  int h, g;                // q-heads, of a kv head
  int window, sinks;
  float scale;             // of the scores, times log2(e)
};

// The keys that some row of a sequence (or of a part of its new tokens) sees, in tiles of kTile tokens: the tiles [0, sink)
// and [low, end).
constexpr int kTile = 32;
struct KeyRange {
  int sink, low, end;
  __device__ __forceinline__ int count() const { return sink + end - low; }
  __device__ __forceinline__ int tile(int i) const { return i < sink ? i : low + i - sink; }
};
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
__device__ __forceinline__ KeyRange keys_of(const AttnCall& a, const SeqRows& r) {
  const int n = min(r.n, a.batch.each);
  if (n == 0) return KeyRange{0, 0, 0};
  return key_range(a, r.length - r.n, r.length - r.n + n - 1);
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
// 16-byte pieces lie.
// =====================================================================================
constexpr int kStepWaves = 4;
constexpr int kStepThreads = kStepWaves * 64;

// Prefix sums over the units of all sequences, 256 at a time.
__device__ __forceinline__ int step_units(const AttnCall& a, int s) {
  if (s >= a.batch.n_seqs) return 0;
  return (keys_of(a, seq_rows(a.batch, s)).count() + kStepWaves - 1) / kStepWaves;
}
struct StepScan {
  int before[kStepThreads + 1];      // units of the sequences in front, within these 256
  int part[kStepWaves];
};
// all threads; returns the units of sequences s0 .. s0 + 255
__device__ __forceinline__ int scan_units(StepScan& m, const AttnCall& a, int s0) {
  const int t = threadIdx.x, wave = t >> 6;
  const int mine = step_units(a, s0 + t);
  const int upto = wave_scan_inclusive(mine);
  __syncthreads();
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
__global__ __launch_bounds__(kStepThreads, D == 256 || MT > 1 ? 1 : 2) void step_kernel(AttnCall a, StepWs ws) {
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
      SeqRows r = seq_rows(a.batch, s);
      r.row0 = uniform(r.row0);
      r.n = uniform(r.n);
      r.length = uniform(r.length);
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
          __amdgpu_buffer_rsrc_t k, v;
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
          const int64_t off = max(x.page, 0) * a.cache.page_stride + (int64_t)(kv * a.cache.page + (tok & (a.cache.page - 1))) * kRow;
          const int bytes = x.page < 0 ? 0 : min(kTile, r.length - tok) * kRow;   // what lies behind the last token reads as zero
          x.k = tile_rsrc(a.cache.k + off, bytes);
          x.v = tile_rsrc(a.cache.v + off, bytes);
          return x;
        };
        u32x4 kw[C::kKLoads];
        uint32_t vw[8][C::kVWords];
        auto load_k = [&](const TileAt& x) __attribute__((always_inline)) {
#pragma unroll
          for (int j = 0; j < C::kKLoads; ++j)
            kw[j] = __builtin_amdgcn_raw_buffer_load_b128(x.k, k_off[j / (C::kKLoads / 2)] + (j % (C::kKLoads / 2)) * 64, 0, 0);
        };
        auto load_v = [&](const TileAt& x) __attribute__((always_inline)) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if constexpr (C::kVWords == 1) {
              vw[j][0] = __builtin_amdgcn_raw_buffer_load_b32(x.v, v_off + j * kRow, 0, 0);
            } else if constexpr (C::kVWords == 2) {
              const auto w = __builtin_amdgcn_raw_buffer_load_b64(x.v, v_off + j * kRow, 0, 0);
              vw[j][0] = w[0];
              vw[j][1] = w[1];
            } else if constexpr (kE4m3) {                 // D = 256: two halves of 128 dims
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                const auto w = __builtin_amdgcn_raw_buffer_load_b64(x.v, v_off + j * kRow + hf * 128, 0, 0);
                vw[j][2 * hf] = w[0];
                vw[j][2 * hf + 1] = w[1];
              }
            } else {
#pragma unroll
              for (int hf = 0; hf < C::kVWords / 4; ++hf) {
                const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(x.v, v_off + j * kRow + hf * 256, 0, 0);
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
        auto v_frag = [&](const uint32_t(&vw)[8][C::kVWords], int d) __attribute__((always_inline)) {
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
          auto sees = [&](int key, int newest, int oldest) __attribute__((always_inline)) {   // by a row in between
            return (now.page >= 0) & (key <= newest) & ((key > oldest - window) | (key < a.sinks));
          };
          bool special = false;
          if (!whole) {
#pragma unroll
            for (int x = 0; x < MT; ++x)
#pragma unroll
              for (int j = 0; j < 8; ++j)
                sc[x][j >> 2][j & 3] = sees(first + 8 * qd + j, row_pos[x], row_pos[x]) ? sc[x][j >> 2][j & 3] : -INFINITY;
            // 0 * NaN is NaN: the values of keys that no row sees become zeros; a key that only some rows see and that
            // holds an infinity or NaN sends the tile to the token by token form below
            uint32_t bad = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const bool some = sees(first + 8 * qd + j, pos_last, pos0);
#pragma unroll
              for (int w = 0; w < C::kVWords; ++w) {
                vw[j][w] = some ? vw[j][w] : 0u;
                if constexpr (kE4m3)                      // a byte 0x7F or 0xFF
                  bad |= ((vw[j][w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
                else                                      // an exponent of ones
                  bad |= ((vw[j][w] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
              }
            }
            special = n > 1 && __builtin_amdgcn_ballot_w64(bad != 0) != 0;
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
          if (!special) {
#pragma unroll
            for (int d = 0; d < C::kDTiles; ++d) {
              const bf16x8 f = v_frag(vw, d);
#pragma unroll
              for (int x = 0; x < MT; ++x) o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pf[x], o[x][d], 0, 0, 0);
            }
          } else {
#pragma unroll 1
            for (int pos = pos0; pos <= pos_last; ++pos) {
              uint32_t seen[8][C::kVWords];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const bool s = sees(first + 8 * qd + j, pos, pos);
#pragma unroll
                for (int w = 0; w < C::kVWords; ++w) seen[j][w] = s ? vw[j][w] : 0u;
              }
#pragma unroll
              for (int d = 0; d < C::kDTiles; ++d) {
                const bf16x8 f = v_frag(seen, d);
#pragma unroll
                for (int x = 0; x < MT; ++x) {
                  const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pf[x], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                  for (int e = 0; e < 4; ++e) o[x][d][e] = row_pos[x] == pos ? o[x][d][e] + y[e] : o[x][d][e];
                }
              }
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

// Joins the parts of a (sequence, kv head) that several workgroups of step_kernel worked on, and writes the rows of
// sequences in which no row sees anything.
template <int D, int MT>
__global__ __launch_bounds__(kStepThreads) void combine_kernel(AttnCall a, StepWs ws, int workgroups) {
  constexpr int kGroups = kStepThreads * 4 / D;           // of threads, each with every kGroups-th part
  __shared__ StepScan scan;
  __shared__ float s_acc[kGroups][D];
  __shared__ float s_sum[kGroups];
  const int s = blockIdx.x, kv = blockIdx.y, t = threadIdx.x, h_kv = a.cache.h_kv;
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
  const SeqRows r = seq_rows(a.batch, s);
  const int R = min(r.n, a.batch.each) * a.g;
  // the workgroup of unit x: the largest w with w * total / W <= x
  const int w0 = units > 0 ? (int)(((first + 1) * W - 1) / total) : 0;
  const int w1 = units > 0 ? (int)(((first + units) * W - 1) / total) : 0;
  if (units > 0 && w0 == w1) return;
  const int group = t / (D / 4), d0 = t % (D / 4) * 4;
  for (int row = 0; row < R; ++row) {
    float top = -INFINITY;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    if (units > 0) {
      for (int w = w0 + t; w <= w1; w += kStepThreads) top = fmaxf(top, ws.stats[(int64_t)(2 * w + (w == w0 ? 1 : 0)) * (16 * MT) + row].x);
      top = wave_max(top);
      __syncthreads();
      if ((t & 63) == 0) s_acc[0][t >> 6] = top;
      __syncthreads();
      top = fmaxf(fmaxf(s_acc[0][0], s_acc[0][1]), fmaxf(s_acc[0][2], s_acc[0][3]));
      const float base = top == -INFINITY ? 0.f : top;
      for (int w = w0 + group; w <= w1; w += kGroups) {
        const int64_t at = (int64_t)(2 * w + (w == w0 ? 1 : 0)) * (16 * MT) + row;
        const float2 st = ws.stats[at];
        const float4 x = *reinterpret_cast<const float4*>(ws.part + at * D + d0);
        const float f = __builtin_amdgcn_exp2f(st.x - base);
        sum += f * st.y;
        acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
      }
      __syncthreads();
      *reinterpret_cast<float4*>(&s_acc[group][d0]) = acc;
      if (d0 == 0) s_sum[group] = sum;
      __syncthreads();
    }
    if (group == 0) {
      if (units > 0) {
#pragma unroll
        for (int x = 1; x < kGroups; ++x) {
          const float4 y = *reinterpret_cast<const float4*>(&s_acc[x][d0]);
          acc.x += y.x; acc.y += y.y; acc.z += y.z; acc.w += y.w;
          sum += s_sum[x];
        }
      }
      const int tok = row / a.g, hq = kv * a.g + row - tok * a.g;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      *reinterpret_cast<uint2*>(a.out.p + (int64_t)hq * a.out.head + (int64_t)(r.row0 + tok) * a.out.token + d0) =
          make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
      if (a.lse != nullptr && d0 == 0)
        a.lse[(int64_t)hq * a.batch.n_tokens + r.row0 + tok] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
  }
}

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

// =====================================================================================
// Dispatch
// =====================================================================================
constexpr int kWorkers = 512;                             // two workgroups a CU

struct AttnPlan {
  int mt;                  // 16-row tiles of the step kernel; 0: too many rows for it
  int workers;
  size_t part_bytes, bytes;
};
static AttnPlan plan_of(const prism_cache* c, const prism_batch* b, int n_q_heads) {
  AttnPlan p = {};
  const int64_t rows = (int64_t)b->max_tokens * (n_q_heads / c->n_kv_heads);
  p.mt = rows <= 16 ? 1 : (rows <= 32 && c->head_dim < 256 ? 2 : 0);
  p.bytes = 256;
  if (p.mt == 0 || b->n_seqs == 0) return p;
  const int64_t units = (int64_t)b->n_seqs * c->n_kv_heads * (((int64_t)b->max_pages * c->page + 127) / 128);
  const int most = c->head_dim == 256 || p.mt > 1 ? kWorkers / 2 : kWorkers;
  p.workers = units < most ? (int)units : most;
  const size_t slots = 2 * (size_t)p.workers * 16 * p.mt;
  p.part_bytes = align_up(slots * c->head_dim * sizeof(float), 256);
  p.bytes = p.part_bytes + align_up(slots * sizeof(float2), 256);
  return p;
}

static int check_attn(const prism_cache* cache, const prism_batch* batch, int n_q_heads) {
  int rc = check_cache(cache);
  if (rc != PRISM_OK || (rc = check_batch(cache, batch)) != PRISM_OK) return rc;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0) return PRISM_ERR_INVALID_ARG;
  if (n_q_heads > 1 << 16 || cache->n_kv_heads > 1 << 15) return PRISM_ERR_UNSUPPORTED;
  return PRISM_OK;
}

template <int D, bool kE4m3, int MT>
static int launch_steps(const AttnCall& a, const AttnPlan& p, char* ws, hipStream_t st) {
  const StepWs w = {reinterpret_cast<float*>(ws), reinterpret_cast<float2*>(ws + p.part_bytes)};
  hipLaunchKernelGGL((step_kernel<D, kE4m3, MT>), dim3(p.workers), dim3(kStepThreads), 0, st, a, w);
  hipLaunchKernelGGL((combine_kernel<D, MT>), dim3(a.batch.n_seqs, a.cache.h_kv), dim3(kStepThreads), 0, st, a, w, p.workers);
  return launch_status();
}
template <int D, bool kE4m3>
static int launch_attn(const AttnCall& a, const AttnPlan& p, char* ws, hipStream_t st) {
  if (p.mt == 1) return launch_steps<D, kE4m3, 1>(a, p, ws, st);
  if constexpr (D < 256)
    if (p.mt == 2) return launch_steps<D, kE4m3, 2>(a, p, ws, st);
  hipLaunchKernelGGL((cache_attn_simple_kernel<D, kE4m3>), dim3(a.batch.n_tokens, a.h), dim3(256), 0, st, a.q, a.out, a.lse, a.cache,
                     a.batch, a.h, a.window, a.sinks, a.scale * kLn2);
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
  *bytes = plan_of(cache, batch, n_q_heads).bytes;
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
  const AttnPlan plan = plan_of(cache, batch, h);
  if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < plan.bytes) return PRISM_ERR_WORKSPACE;
  const float scale = params->scale > 0.f ? params->scale : 1.f / sqrtf((float)d);
  const AttnCall a = {rows_of(q), rows_of(out), lse, cache_view(cache), batch_view(batch), h, h / cache->n_kv_heads,
                      params->window, params->sinks, scale * kLog2e};
  const bool e4m3 = cache->dtype == PRISM_CACHE_E4M3;
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (d) {
    case 64: return launch_for<64>(e4m3, a, plan, ws, st);
    case 128: return launch_for<128>(e4m3, a, plan, ws, st);
    default: return launch_for<256>(e4m3, a, plan, ws, st);
  }
}
