// gfx950 (MI355X, CDNA4) kernels of the 8-bit cache: writing it, and attention over it.
//
// Formats. A page holds 128 tokens of every key head: K codes [token][d], V codes [d][token], both
// e4m3 (OCP), with one fp32 scale per page and head for K and one for V. V lies transposed so that
// the matrix cores' operand of O^T += V^T P^T (16 rows of d, 8 consecutive tokens per lane) is one
// plain load. Written scales are powers of two: e4m3 keeps 4 significant bits at any magnitude, so
// a power of two costs nothing except at the ends of the range, and when a later token raises a
// page's scale the codes it held move by whole exponents (exactly, but for those that become
// subnormal).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <stdint.h>

#include "block_launch.h"
#include "tile_common.h"

namespace ta {
namespace {

constexpr int kThreadsC = 256;
constexpr float kMaxCode = 448.f;  // the largest e4m3 magnitude
constexpr int kMinExp = -100, kMaxExp = 120;

// ---------------------------------------------------------------------------------------------
// write

// The least e in [kMinExp, kMaxExp] with amax <= 448 * 2^e; amax > 0 finite, given by its bits.
// amax = 1.m * 2^x and 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(uint32_t bits) {
  if (bits == 0) return kMinExp;
  const int x = (int)(bits >> 23) - 127;
  const int e = (bits & 0x7fffffu) <= 0x600000u ? x - 8 : x - 7;
  return min(max(e, kMinExp), kMaxExp);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// e4m3 code of x: nearest, ties to even; infinities become +-448, NaN stays NaN.
__device__ __forceinline__ uint32_t code_of(float x) {
  const float y = __builtin_amdgcn_fmed3f(x, -kMaxCode, kMaxCode);
  const uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 0xffu;
  return x != x ? 0x7fu : c;
}
__device__ __forceinline__ float value_of(uint32_t code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }

// One workgroup writes K (blockIdx.z = 0) or V (1) of one (sequence, key head, touched page).
template <int D>
__global__ __launch_bounds__(kThreadsC) void cache_write_kernel(const CacheWriteArgs a) {
  constexpr int kPieces = D / 8;  // 16-byte pieces of a token's bf16 row
  __shared__ uint32_t s_max[kThreadsC / 64];
  __shared__ uint8_t s_codes[D * (kBlock + 4)];  // V: codes [d][token], rows padded against bank conflicts
  const int b = blockIdx.y / a.Hkv, h = blockIdx.y - b * a.Hkv;
  const bool is_v = blockIdx.z != 0;
  const int64_t len = max(a.lens[b], 0);
  const int n = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
  const int64_t slot = len / kBlock + blockIdx.x;
  if (slot >= a.max_pages) return;
  // Page positions [t0, t1) receive new tokens, the first of them token `src`.
  const int64_t pos0 = slot * kBlock;
  const int t0 = (int)max(len - pos0, (int64_t)0);
  const int t1 = (int)min(len + n - pos0, (int64_t)kBlock);
  if (t1 <= t0) return;
  const int page = a.table[(size_t)b * a.max_pages + slot];
  if (page < 0 || page >= a.n_pages) return;
  const size_t ph = (size_t)page * a.Hkv + h;
  const uint16_t* x = (is_v ? a.v : a.k) + (((size_t)b * a.Hkv + h) * a.N + (size_t)(pos0 + t0 - len)) * D;
  uint8_t* codes = (is_v ? a.v_pages : a.k_pages) + ph * kBlock * D;
  float* scale = (is_v ? a.v_scales : a.k_scales) + ph;
  const int tid = threadIdx.x;
  const int n_pieces = (t1 - t0) * kPieces;

  // The largest finite magnitude of the new tokens: bf16 bits without the sign order as integers.
  uint32_t most = 0;
  for (int p = tid; p < n_pieces; p += kThreadsC) {
    const u32x4 w = load16(x + 8 * (size_t)p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t lo = w[e] & 0x7fffu, hi = (w[e] >> 16) & 0x7fffu;
      most = max(most, lo < 0x7f80u ? lo : 0u);
      most = max(most, hi < 0x7f80u ? hi : 0u);
    }
  }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, s));
  if ((tid & 63) == 0) s_max[tid >> 6] = most;
  const float s_old = *scale;
  __syncthreads();
  most = 0;
#pragma unroll
  for (int w = 0; w < kThreadsC / 64; ++w) most = max(most, s_max[w]);
  float s_new = pow2(scale_exponent(most << 16));
  if (t0 > 0) s_new = fmaxf(s_old, s_new);
  const float inv = 1.f / s_new;  // exact: a power of two, unless the page's own scale was none

  if (t0 > 0 && s_new != s_old) {
    // The page's old tokens under the larger scale.
    const float ratio = s_old * inv;
    for (int p = tid; p < t0 * D; p += kThreadsC) {
      uint8_t* c = is_v ? codes + (size_t)(p / t0) * kBlock + p % t0 : codes + p;
      *c = (uint8_t)code_of(value_of(*c) * ratio);
    }
  }
  if (!is_v) {
    for (int p = tid; p < n_pieces; p += kThreadsC) {
      const u32x4 w = load16(x + 8 * (size_t)p);
      u32x2 c = {0u, 0u};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e / 2] |= code_of(__uint_as_float(w[e] << 16) * inv) << (16 * (e % 2));
        c[e / 2] |= code_of(__uint_as_float(w[e] & 0xffff0000u) * inv) << (16 * (e % 2) + 8);
      }
      *reinterpret_cast<u32x2*>(codes + (size_t)t0 * D + 8 * (size_t)p) = c;
    }
  } else {
    constexpr int kRow = kBlock + 4;
    for (int p = tid; p < n_pieces; p += kThreadsC) {
      const u32x4 w = load16(x + 8 * (size_t)p);
      const int t = t0 + p / kPieces, d0 = 8 * (p % kPieces);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s_codes[(d0 + 2 * e) * kRow + t] = (uint8_t)code_of(__uint_as_float(w[e] << 16) * inv);
        s_codes[(d0 + 2 * e + 1) * kRow + t] = (uint8_t)code_of(__uint_as_float(w[e] & 0xffff0000u) * inv);
      }
    }
    __syncthreads();
    // Whole dwords of four tokens where all four are new, single bytes at the ends.
    for (int p = tid; p < D * (kBlock / 4); p += kThreadsC) {
      const int d0 = p / (kBlock / 4), t = 4 * (p % (kBlock / 4));
      if (t >= t1 || t + 4 <= t0) continue;
      uint8_t* dst = codes + (size_t)d0 * kBlock + t;
      const uint8_t* from = s_codes + d0 * kRow + t;
      if (t >= t0 && t + 4 <= t1) {
        *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(from);
      } else {
        for (int y = max(t0 - t, 0); y < min(t1 - t, 4); ++y) dst[y] = from[y];
      }
    }
  }
  if (tid == 0 && s_new != s_old) *scale = s_new;
}

// ---------------------------------------------------------------------------------------------
// attention
//
// The cache's bytes bound this: a decoding step reads every code once and does 4 G N operations a
// byte. Tiles of 64 tokens go from memory into registers, one tile ahead, as the operands of
// v_mfma_f32_16x16x32_bf16 (A: lane l holds row l % 16 and the k indices 8 (l / 16) .. + 7; B the
// same with columns; C: column l % 16, rows 4 (l / 16) + j):
//   S^T = K Q^T. The matrix instruction adds over k in any order, so a lane's 16 bytes of a K row,
//   dims 64 c + 16 g .. + 15 (g = l / 16), serve two instructions, and q is laid out alike. Which
//   token a row of A holds is free too: row r of instruction group i (of 4) is token
//   16 (r / 4) + 4 i + r % 4, which puts tokens 16 g .. 16 g + 15 of the tile's scores into lane
//   group g, in order: exactly the P^T operand of
//   O^T += V^T P^T, whose V operand is 16 bytes of a V row (tokens 16 g .. + 15).
// e4m3 codes become bf16 exactly (v_cvt_scalef32_pk_bf16_fp8); the page's K scale multiplies the
// scores and its V scale the weights, in fp32. The row sums add the weights before they are rounded
// to bf16 for the matrix cores.
//
// The pages of all sequences and key heads form one line that `workers` workgroups share evenly,
// whatever the lengths: a workgroup runs the (sequence, head) segments its stretch meets, writes
// those it has alone, and leaves a partial result (at most two) of those it shares; a second
// kernel joins them in the order of the pages.


// The line of all segments' pages. Segment order: entry i of lens, then (where all heads share an
// entry) the key heads. Every wave finds its place by itself, 64 entries at a time.
struct Place {
  int64_t total;  // pages of the line
  int64_t start;  // of entry `entry`, pages of the line before it
  int entry;      // the entry that holds the asked page (or the asked entry)
};
__device__ __forceinline__ int cache_len(const CacheAttnArgs& a, int i) {
  return (int)min((int64_t)max(a.lens[i], 0), (int64_t)a.max_pages * kBlock);
}
__device__ __forceinline__ int pages_of(int len) { return (len + kBlock - 1) / kBlock; }

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x += __shfl_xor((long long)x, s);
  return x;
}
__device__ __forceinline__ int64_t line_total(const CacheAttnArgs& a, int entries, int per) {
  const int lane = threadIdx.x & 63;
  int64_t n = 0;
  for (int i = lane; i < entries; i += 64) n += pages_of(cache_len(a, i));
  return wave_sum(n) * per;
}
// The entry that holds page `at` of the line (at < total), and the line's pages before it.
__device__ __forceinline__ Place find_page(const CacheAttnArgs& a, int entries, int per, int64_t total, int64_t at) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int i0 = 0; i0 < entries; i0 += 64) {
    const int64_t own = i0 + lane < entries ? (int64_t)pages_of(cache_len(a, i0 + lane)) * per : 0;
    int64_t upto = own;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int64_t y = __shfl_up((long long)upto, s);
      if (lane >= s) upto += y;
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto > at);
    if (past) {
      const int src = __ffsll((unsigned long long)past) - 1;
      return Place{total, before + __shfl((long long)(upto - own), src), i0 + src};
    }
    before += __shfl((long long)upto, 63);
  }
  return Place{total, total, entries};
}
// The first page of the line that worker w of W takes, and the worker that takes page x.
__device__ __forceinline__ int64_t worker_start(int64_t total, int w, int W) { return total * w / W; }
__device__ __forceinline__ int worker_of(int64_t total, int64_t x, int W) {
  return (int)(((x + 1) * W + total - 1) / total) - 1;
}

// max and sum over the four lane groups that hold one query row's tokens.
__device__ __forceinline__ float group_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float group_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Eight e4m3 codes as bf16, exactly.
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

constexpr int kTile = 64;      // tokens of a wave's tile: half a page
constexpr float kNoRef = -1e30f;  // a running maximum before the first token (base-2 logits)

// One tile's codes and scales in a lane's registers; page < 0: no tile.
template <int D>
struct CacheTile {
  uint32_t k[4][D / 16];
  u32x4 v[D / 16];
  float ks, vs;
  int page;
  __device__ __forceinline__ void load(const CacheAttnArgs& a, int p, int h, int half, int lane) {
    page = p;
    if (p < 0) return;
    const size_t ph = (size_t)p * a.Hkv + h;
    ks = a.k_scales[ph];
    vs = a.v_scales[ph];
    const int n = lane & 15, g = lane >> 4;
    const uint8_t* kb = a.k_pages + (ph * kBlock + half * kTile) * D + (16 * (n >> 2) + (n & 3)) * D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint8_t* row = kb + 4 * i * D;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(row + 64 * c + 16 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) k[i][4 * c + e] = w[e];
      }
      if constexpr (D % 64 != 0) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(row + D / 64 * 64 + 8 * g);
        k[i][D / 16 - 2] = w[0];
        k[i][D / 16 - 1] = w[1];
      }
    }
    const uint8_t* vb = a.v_pages + ph * kBlock * D + n * kBlock + half * kTile + 16 * g;
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb) v[mb] = *reinterpret_cast<const u32x4*>(vb + 16 * mb * kBlock);
  }
};

// The first dim of the 8 that lane group g holds of 32-wide slice m of q and K.
template <int D>
__device__ __forceinline__ int slice_dim(int m, int g) {
  return m < D / 64 * 2 ? 64 * (m / 2) + 16 * g + 8 * (m % 2) : D / 64 * 64 + 8 * g;
}

template <int D, int RB>
__global__ __launch_bounds__(kThreadsC, 2) void cache_attn_kernel(const CacheAttnArgs a) {
  constexpr int kRows = 16 * RB, kWaves = kThreadsC / 64, kMb = D / 16, kSl = D / 32;
  __shared__ float s_o[kWaves][kRows][D + 4];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 15, g = lane >> 4;
  const int entries = a.per_head ? a.B * a.Hkv : a.B, per = a.per_head ? 1 : a.Hkv;
  const int w = blockIdx.x, row0 = blockIdx.y * kRows, rows = a.G * a.N;

  const int64_t total = line_total(a, entries, per);
  const int64_t lo = worker_start(total, w, a.workers), hi = worker_start(total, w + 1, a.workers);
  if (lo >= hi) return;
  const Place pl = find_page(a, entries, per, total, lo);
  int entry = __builtin_amdgcn_readfirstlane(pl.entry);
  int len = __builtin_amdgcn_readfirstlane(cache_len(a, entry));
  int pages = pages_of(len);
  int head = (int)((lo - pl.start) / pages);
  int64_t seg0 = pl.start + (int64_t)head * pages;  // the line's page where the segment starts

  int64_t at = lo;
  while (at < hi) {
    const int h = a.per_head ? entry % a.Hkv : head, b = a.per_head ? entry / a.Hkv : entry;
    const int p0 = (int)(at - seg0), p1 = (int)min((int64_t)pages, hi - seg0);
    const int32_t* table = a.table + (size_t)entry * a.max_pages;
    const size_t q_row = ((size_t)b * a.H + (size_t)h * a.G) * a.N;  // rows of the group lie together

    bf16x8 qf[RB][kSl];
    int end[RB];  // tokens this lane's row attends to
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = row0 + 16 * rb + n;
      end[rb] = r < rows ? len - (a.N - 1) + r % a.N : 0;
#pragma unroll
      for (int m = 0; m < kSl; ++m) {
        u32x4 x = {0u, 0u, 0u, 0u};
        if (r < rows) x = load16(a.q + (q_row + r) * D + slice_dim<D>(m, g));
        qf[rb][m] = as_bf16x8(x);
      }
    }
    f32x4 o[RB][kMb];
    float m_ref[RB], l_run[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m_ref[rb] = kNoRef;
      l_run[rb] = 0.f;
#pragma unroll
      for (int mb = 0; mb < kMb; ++mb) o[rb][mb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Tiles wave, wave + 4, ... of pages [p0, p1), those that hold a token.
    const int t_end = min(2 * p1, (len + kTile - 1) / kTile);
    auto page_of = [&](int t) {
      if (t >= t_end) return -1;
      const int p = table[t >> 1];
      return p < a.n_pages ? p : -1;  // no page: its tokens are not read
    };
    auto step = [&](CacheTile<D>& cur, int t) {
      if (cur.page < 0) return;
      const int tok0 = t * kTile;
      if (tok0 + kTile > len) {  // codes behind the last token may be NaN: clear them in V
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int left = len - (tok0 + 16 * g + 4 * e);
          const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
          for (int mb = 0; mb < kMb; ++mb) cur.v[mb][e] &= keep;
        }
      }
      f32x4 s[RB][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int m = 0; m < kSl; ++m) {
          const bf16x8 kf = widen8(cur.k[i][2 * m], cur.k[i][2 * m + 1]);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            s[rb][i] = mfma16(kf, qf[rb][m], m == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[rb][i]);
        }
      const float c = a.c * cur.ks;
      bf16x8 pf[RB][2];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[rb][i] *= c;
        if (tok0 + kTile > len - (a.N - 1)) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (tok0 + 16 * g + 4 * i + j >= end[rb]) s[rb][i][j] = -INFINITY;
        }
        float mx = s[rb][0][0];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) mx = fmaxf(mx, s[rb][i][j]);
        const float m_new = fmaxf(m_ref[rb], group_max(mx));
        if (__builtin_amdgcn_ballot_w64(m_new > m_ref[rb])) {
          const float alpha = fast_exp2(m_ref[rb] - m_new);
          l_run[rb] *= alpha;
#pragma unroll
          for (int mb = 0; mb < kMb; ++mb) o[rb][mb] *= alpha;
          m_ref[rb] = m_new;
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float p = fast_exp2(s[rb][i][j] - m_ref[rb]);
            sum += p;
            pf[rb][i / 2][4 * (i % 2) + j] = (__bf16)(p * cur.vs);
          }
        l_run[rb] += sum;
      }
#pragma unroll
      for (int mb = 0; mb < kMb; ++mb)
#pragma unroll
        for (int c2 = 0; c2 < 2; ++c2) {
          const bf16x8 vf = widen8(cur.v[mb][2 * c2], cur.v[mb][2 * c2 + 1]);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) o[rb][mb] = mfma16(vf, pf[rb][c2], o[rb][mb]);
        }
    };
    int t = 2 * p0 + wave;
    CacheTile<D> ta, tb;
    ta.load(a, page_of(t), h, t & 1, lane);
    int next = page_of(t + kWaves);
    for (; t < t_end; t += 2 * kWaves) {
      tb.load(a, next, h, (t + kWaves) & 1, lane);
      next = page_of(t + 2 * kWaves);
      step(ta, t);
      ta.load(a, next, h, (t + 2 * kWaves) & 1, lane);
      next = page_of(t + 3 * kWaves);
      step(tb, t + kWaves);
    }

    // The waves' states join in LDS.
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float l = group_sum(l_run[rb]);
      if (g == 0) {
        s_m[wave][16 * rb + n] = m_ref[rb];
        s_l[wave][16 * rb + n] = l;
      }
#pragma unroll
      for (int mb = 0; mb < kMb; ++mb) *reinterpret_cast<f32x4*>(&s_o[wave][16 * rb + n][16 * mb + 4 * g]) = o[rb][mb];
    }
    __syncthreads();
    const bool alone = p0 == 0 && p1 == pages;
    const int slot = 2 * w + (at == lo ? 0 : 1);
    float* part = a.part + ((size_t)blockIdx.y * 2 * a.workers + slot) * kRows * (D + 2);
    for (int i = tid; i < kRows * (D / 4); i += kThreadsC) {
      const int r = i / (D / 4), d0 = 4 * (i % (D / 4));
      if (row0 + r >= rows) continue;
      float m = s_m[0][r];
#pragma unroll
      for (int x = 1; x < kWaves; ++x) m = fmaxf(m, s_m[x][r]);
      float l = 0.f;
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        const float f = fast_exp2(s_m[x][r] - m);
        l += f * s_l[x][r];
        y += f * *reinterpret_cast<const f32x4*>(&s_o[x][r][d0]);
      }
      y *= l > 0.f ? 1.f / l : 0.f;
      const float lse2 = l > 0.f ? m + __builtin_amdgcn_logf(l) : -INFINITY;
      if (alone) {
        *reinterpret_cast<u32x2*>(a.out + (q_row + row0 + r) * D + d0) =
            __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
        if (a.lse && d0 == 0) a.lse[q_row + row0 + r] = lse2 * 0.69314718055994531f;
      } else {
        float* pr = part + (size_t)r * (D + 2);
        *reinterpret_cast<f32x2*>(pr + d0) = f32x2{y[0], y[1]};
        *reinterpret_cast<f32x2*>(pr + d0 + 2) = f32x2{y[2], y[3]};
        if (d0 == 0) pr[D] = lse2;
      }
    }
    __syncthreads();

    at = seg0 + p1;
    if (p1 == pages) {  // the next segment with pages
      seg0 += pages;
      if (++head == per) {
        head = 0;
        pages = 0;
        while (pages == 0 && ++entry < entries) {
          len = __builtin_amdgcn_readfirstlane(cache_len(a, entry));
          pages = pages_of(len);
        }
      }
    }
  }
}

// Joins the partial results of a segment that several workers share, in the order of its pages;
// a segment without tokens gets its zeros here.
template <int D, int RB>
__global__ __launch_bounds__(kThreadsC) void cache_merge_kernel(const CacheAttnArgs a) {
  constexpr int kRows = 16 * RB;
  const int entries = a.per_head ? a.B * a.Hkv : a.B, per = a.per_head ? 1 : a.Hkv;
  const int b = blockIdx.x / a.Hkv, h = blockIdx.x - b * a.Hkv;
  const int entry = a.per_head ? (int)blockIdx.x : b;
  const int row0 = blockIdx.y * kRows, rows = a.G * a.N;
  const int lane = threadIdx.x & 63;
  const int pages = pages_of(cache_len(a, entry));
  const int64_t total = line_total(a, entries, per);
  int64_t before = 0;
  for (int i = lane; i < entry; i += 64) before += pages_of(cache_len(a, i));
  const int64_t s0 = wave_sum(before) * per + (a.per_head ? 0 : (int64_t)h * pages);
  int w0 = 0, w1 = -1;
  if (pages > 0) {
    w0 = worker_of(total, s0, a.workers);
    w1 = worker_of(total, s0 + pages - 1, a.workers);
    if (w0 == w1) return;  // that worker wrote the rows
  }
  const size_t q_row = ((size_t)b * a.H + (size_t)h * a.G) * a.N;
  const float* parts = a.part + (size_t)blockIdx.y * 2 * a.workers * kRows * (D + 2);
  auto row_of = [&](int w, int r) {
    return parts + ((size_t)(2 * w + (worker_start(total, w, a.workers) < s0 ? 1 : 0)) * kRows + r) * (D + 2);
  };
  auto empty = [&](int w) {
    return worker_start(total, w, a.workers) == worker_start(total, w + 1, a.workers);
  };
  for (int i = threadIdx.x; i < kRows * (D / 4); i += kThreadsC) {
    const int r = i / (D / 4), d0 = 4 * (i % (D / 4));
    if (row0 + r >= rows) continue;
    float m = -INFINITY;
    for (int w = w0; w <= w1; ++w)
      if (!empty(w)) m = fmaxf(m, row_of(w, r)[D]);
    float l = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    if (m > -INFINITY) {
      for (int w = w0; w <= w1; ++w) {
        if (empty(w)) continue;
        const float* pr = row_of(w, r);
        const float f = fast_exp2(pr[D] - m);
        const f32x2 u = *reinterpret_cast<const f32x2*>(pr + d0), v = *reinterpret_cast<const f32x2*>(pr + d0 + 2);
        l += f;
        y += f * f32x4{u[0], u[1], v[0], v[1]};
      }
      y *= 1.f / l;
    }
    *reinterpret_cast<u32x2*>(a.out + (q_row + row0 + r) * D + d0) =
        __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
    if (a.lse && d0 == 0)
      a.lse[q_row + row0 + r] = m > -INFINITY ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f : -INFINITY;
  }
}

template <int D>
hipError_t cache_attn_for(const CacheAttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.workers, (unsigned)a.row_blocks), segs((unsigned)(a.B * a.Hkv), (unsigned)a.row_blocks);
  if (cache_rows_per_pass(a.G * a.N) == 16) {
    cache_attn_kernel<D, 1><<<grid, kThreadsC, 0, s>>>(a);
    cache_merge_kernel<D, 1><<<segs, kThreadsC, 0, s>>>(a);
  } else {
    cache_attn_kernel<D, 2><<<grid, kThreadsC, 0, s>>>(a);
    cache_merge_kernel<D, 2><<<segs, kThreadsC, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

int cache_rows_per_pass(int rows) { return rows <= 16 ? 16 : 32; }

hipError_t launch_cache_write(const CacheWriteArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((kBlock - 1 + (int64_t)a.N + kBlock - 1) / kBlock), (unsigned)(a.B * a.Hkv), 2);
  if (a.d == 64) cache_write_kernel<64><<<grid, kThreadsC, 0, stream>>>(a);
  else if (a.d == 96) cache_write_kernel<96><<<grid, kThreadsC, 0, stream>>>(a);
  else cache_write_kernel<128><<<grid, kThreadsC, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, hipStream_t stream) {
  if (a.d == 64) return cache_attn_for<64>(a, stream);
  if (a.d == 96) return cache_attn_for<96>(a, stream);
  return cache_attn_for<128>(a, stream);
}

}  // namespace ta
