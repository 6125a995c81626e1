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

#include <type_traits>

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

// e4m3 codes of two numbers in the low (or high) half of a word: nearest, ties to even; infinities become
// +-448, NaN stays NaN.
template <bool HIGH>
__device__ __forceinline__ uint32_t code_pair(float x, float y, uint32_t word) {
  const float a = __builtin_amdgcn_fmed3f(x, -kMaxCode, kMaxCode), b = __builtin_amdgcn_fmed3f(y, -kMaxCode, kMaxCode);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x != x ? x : a, y != y ? y : b, (int)word, HIGH);
}
__device__ __forceinline__ float bf16_at(u32x4 w, int e) {
  return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
}

// Bound by the bytes, and for single tokens by the latency of its loads: table and length, scale and
// token, then the codes. Two prompts of 8191 tokens, 8 heads of 128: 23.4 us for 101 MB (4.3 TB/s; a large
// copy 5.0); one token of 32 sequences: 5.3 us.
// One workgroup writes K (blockIdx.z = 0) or V (1) of one (sequence, key head, touched page). A thread
// holds 16-byte pieces (8 dims) of four tokens in a row, read once: the page's maximum needs them all
// before the first can be rounded. K codes go out as they lie, V's through LDS.
template <int D>
__global__ __launch_bounds__(kThreadsC) void cache_write_kernel(const CacheWriteArgs a) {
  constexpr int kPieces = D / 8, kPer = (kBlock / 4 * kPieces + kThreadsC - 1) / kThreadsC;
  constexpr int kRow = kBlock + 16;  // bytes of a V row in LDS: rows of 16-byte pieces, on different banks
  __shared__ uint32_t s_max[kThreadsC / 64];
  __shared__ __attribute__((aligned(16))) uint8_t s_codes[D * kRow];
  const int b = blockIdx.y / a.Hkv, h = blockIdx.y - b * a.Hkv;
  const bool is_v = blockIdx.z != 0;
  const int64_t len = max(a.lens[b], 0);
  const int n = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
  const int64_t slot = len / kBlock + blockIdx.x;
  if (slot >= a.max_pages) return;
  // Page positions [t0, t1) receive new tokens, the first of them token pos0 + t0 - len of the call.
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
  const int g0 = t0 / 4 * kPieces, g1 = (t1 + 3) / 4 * kPieces;  // items that hold new tokens

  // The largest finite magnitude of the new tokens: bf16 bits without the sign order as integers.
  const float s_old = *scale;
  u32x4 w[kPer][4];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int item = g0 + tid + kThreadsC * i, t = item / kPieces * 4, d0 = item % kPieces * 8;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      w[i][y] = u32x4{0u, 0u, 0u, 0u};
      if (item < g1 && t + y >= t0 && t + y < t1) w[i][y] = load16(x + (size_t)(t + y - t0) * D + d0);
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = w[i][y][e] & 0x7fffu, hi = (w[i][y][e] >> 16) & 0x7fffu;
        most = max(most, lo < 0x7f80u ? lo : 0u);
        most = max(most, hi < 0x7f80u ? hi : 0u);
      }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, s));
  if ((tid & 63) == 0) s_max[tid >> 6] = most;
  __syncthreads();
  most = 0;
#pragma unroll
  for (int y = 0; y < kThreadsC / 64; ++y) most = max(most, s_max[y]);
  float s_new = pow2(scale_exponent(most << 16));
  if (t0 > 0) s_new = fmaxf(s_old, s_new);
  const float inv = 1.f / s_new;  // exact: a power of two

  if (t0 > 0 && s_new != s_old) {
    // The page's old tokens under the larger scale, 16 codes at a time: of K the first t0 rows, of V the
    // first t0 of every row (the codes behind them stay as they are).
    const float ratio = s_old * inv;
    constexpr int kVecs = kBlock / 16;
    const int vecs = is_v ? D * kVecs : t0 * (D / 16);
    for (int p = tid; p < vecs; p += kThreadsC) {
      const int old = is_v ? min(max(t0 - p % kVecs * 16, 0), 16) : 16;  // codes of these 16 to move
      if (old == 0) continue;
      u32x4 c = *reinterpret_cast<const u32x4*>(codes + 16 * (size_t)p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = (int)c[e];
        uint32_t y = code_pair<false>(__builtin_amdgcn_cvt_f32_fp8(v, 0) * ratio,
                                      __builtin_amdgcn_cvt_f32_fp8(v, 1) * ratio, 0u);
        y = code_pair<true>(__builtin_amdgcn_cvt_f32_fp8(v, 2) * ratio, __builtin_amdgcn_cvt_f32_fp8(v, 3) * ratio, y);
        const int left = old - 4 * e;
        const uint32_t keep = left >= 4 ? 0u : left <= 0 ? ~0u : ~0u << (8 * left);
        c[e] = (y & ~keep) | (c[e] & keep);
      }
      *reinterpret_cast<u32x4*>(codes + 16 * (size_t)p) = c;
    }
    if (is_v) __syncthreads();  // new tokens may share 16 codes with old ones
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int item = g0 + tid + kThreadsC * i, t = item / kPieces * 4, d0 = item % kPieces * 8;
    if (item >= g1) continue;
    if (!is_v) {
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if (t + y < t0 || t + y >= t1) continue;
        u32x2 c = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          c[e] = code_pair<false>(bf16_at(w[i][y], 4 * e) * inv, bf16_at(w[i][y], 4 * e + 1) * inv, 0u);
          c[e] = code_pair<true>(bf16_at(w[i][y], 4 * e + 2) * inv, bf16_at(w[i][y], 4 * e + 3) * inv, c[e]);
        }
        *reinterpret_cast<u32x2*>(codes + (size_t)(t + y) * D + d0) = c;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t c = code_pair<false>(bf16_at(w[i][0], e) * inv, bf16_at(w[i][1], e) * inv, 0u);
        c = code_pair<true>(bf16_at(w[i][2], e) * inv, bf16_at(w[i][3], e) * inv, c);
        *reinterpret_cast<uint32_t*>(s_codes + (d0 + e) * kRow + t) = c;
      }
    }
  }
  if (is_v) {
    __syncthreads();
    // 16 codes at a time where all are new, single ones at the ends.
    const int v0 = t0 / 16, nv = (t1 + 15) / 16 - v0;
    for (int p = tid; p < D * nv; p += kThreadsC) {
      const int d0 = p / nv, t = 16 * (v0 + p - d0 * nv);
      uint8_t* dst = codes + (size_t)d0 * kBlock + t;
      const uint8_t* from = s_codes + d0 * kRow + t;
      if (t >= t0 && t + 16 <= t1) {
        *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>(from);
      } else {
        for (int y = max(t0 - t, 0); y < min(t1 - t, 16); ++y) dst[y] = from[y];
      }
    }
  }
  if (tid == 0 && s_new != s_old) *scale = s_new;
}

// ---------------------------------------------------------------------------------------------
// attention
//
// The cache's bytes bound this: a decoding step reads every code once and does 4 G N operations a
// byte (32 sequences of 512 to 65536 tokens, 8 key heads of 128: 185 to 188 us for 0.92 GB, 4.9 TB/s; a
// large copy reaches 5.0). A wave takes a page at a time, its codes from memory straight into registers, one page ahead,
// as the operands of v_mfma_f32_16x16x32_bf16 (A: lane l holds row l % 16 and the k indices 8 (l / 16) .. + 7; B the
// same with columns; C: column l % 16, rows 4 (l / 16) + j):
//   S^T = K Q^T. The matrix instruction adds over k in any order, so a lane's 16 bytes of a K row,
//   dims 64 c + 16 g .. + 15 (g = l / 16), serve two instructions, and q is laid out alike. Which
//   token a row of A holds is free too: in each half of 64 tokens row r of instruction group i (of
//   4) is token 16 (r / 4) + 4 i + r % 4, which puts the scores of tokens 16 g .. 16 g + 15 into lane
//   group g, in order: exactly the P^T operand of
//   O^T += V^T P^T, whose V operand is 16 bytes of a V row (tokens 16 g .. + 15).
// e4m3 codes become bf16 exactly (v_cvt_scalef32_pk_bf16_fp8); the page's K scale multiplies the
// scores and its V scale the weights, in fp32. The row sums add the weights before they are rounded
// to bf16, times the V scale, for the matrix cores (which take fp32 at a sixteenth of the rate): that
// rounding moves the error against 64 bits, the results' own in it, from 1.7e-3 to 2.2e-3.
//
// The pages of all sequences and key heads form one line that `workers` workgroups share evenly,
// whatever the lengths: a workgroup runs the (sequence, head) segments its stretch meets, writes
// those it has alone, and leaves a partial result (at most two) of those it shares; a second
// kernel joins them in the order of the pages.


// A quotient of numbers that are the same in every lane, in a scalar register (the division itself runs
// on the vector ALU; left there, it would make every address and branch behind it a lane's own).
__device__ __forceinline__ int scalar_div(int x, int y) {
  return __builtin_amdgcn_readfirstlane((int)((uint32_t)x / (uint32_t)y));
}

// The line of all segments, each kSegment + its pages long (below 2^31, checked by the host): what a
// segment's start and end cost a workgroup is about kSegment pages' time (32 sequences of 4 to 512
// pages: 208 us with 0, 188 with 3). Segment order: entry i of lens, then (where all heads share an
// entry) the key heads. Worker w takes line / workers, the first line % workers ones one more. Every
// wave finds its place by itself, 64 entries at a time.
constexpr int kSegment = kCacheSegment;
using ScalarInts = const __attribute__((address_space(4))) int32_t*;    // read with scalar loads
using ScalarFloats = const __attribute__((address_space(4))) float*;

__device__ __forceinline__ int cache_len(const CacheAttnArgs& a, int i) {
  return (int)min((int64_t)max(a.lens[i], 0), (int64_t)a.max_pages * kBlock);
}
__device__ __forceinline__ int pages_of(int len) { return (int)(((uint32_t)len + kBlock - 1) / kBlock); }
// A segment's length on the line; one without pages has none.
__device__ __forceinline__ int extent_of(int pages) { return pages > 0 ? kSegment + pages : 0; }

struct Line {
  int entries, per;  // entries of lens, segments of an entry
  int total;         // its length
  int each, more;    // every worker's part, workers with one more
  __device__ __forceinline__ Line(const CacheAttnArgs& a, bool measure = true) {
    entries = a.per_head ? a.B * a.Hkv : a.B;
    per = a.per_head ? 1 : a.Hkv;
    total = each = more = 0;
    if (!measure) return;
    int n = 0;
    for (int i = threadIdx.x & 63; i < entries; i += 64) n += extent_of(pages_of(cache_len(a, i)));
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) n += __shfl_xor(n, s);
    total = __builtin_amdgcn_readfirstlane(n) * per;
    each = scalar_div(total, a.workers);
    more = total - each * a.workers;
  }
  __device__ __forceinline__ int start(int w) const { return w * each + min(w, more); }
  // The worker that takes place x of the line, x < total.
  __device__ __forceinline__ int worker(int x) const {
    const int y = x - more * (each + 1);
    return y < 0 ? scalar_div(x, each + 1) : more + scalar_div(y, each);
  }
  // The entry that holds place `at` (at < total), and where it starts.
  __device__ __forceinline__ int entry_of(const CacheAttnArgs& a, int at, int& before) const {
    const int lane = threadIdx.x & 63;
    before = 0;
    for (int i0 = 0; i0 < entries; i0 += 64) {
      const int own = i0 + lane < entries ? extent_of(pages_of(cache_len(a, i0 + lane))) * per : 0;
      int upto = own;
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const int y = __shfl_up(upto, s);
        if (lane >= s) upto += y;
      }
      const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto > at);
      if (past) {
        const int src = __ffsll((unsigned long long)past) - 1;
        before = __builtin_amdgcn_readfirstlane(before + __shfl(upto - own, src));
        return __builtin_amdgcn_readfirstlane(i0 + src);
      }
      before = __builtin_amdgcn_readfirstlane(before + __shfl(upto, 63));
    }
    return entries;
  }
};

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
// A one in the lowest bit of every byte that is a NaN code (0x7f, 0xff).
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u; }
// The bytes of a word that come before byte `left`.
__device__ __forceinline__ uint32_t bytes_before(int left) {
  return left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
}
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

constexpr float kNoRef = -1e30f;  // a running maximum before the first token (base-2 logits)

// A page's codes in a lane's registers, by halves of 64 tokens. Base addresses are the same in every
// lane (scalar registers), lanes add a 32-bit offset that no page changes. Both halves of a V row (a
// 128-byte line) are read one after the other: with 64 tokens a wave the second half came from memory
// again a third of the time (1.04 GB fetched for 0.88).
template <int D>
struct KeyPage {
  uint32_t k[8][D / 16];
  __device__ __forceinline__ void load(const uint8_t* page, int lane) {
    const int n = lane & 15, g = lane >> 4;
    const uint32_t at = (uint32_t)((16 * (n >> 2) + (n & 3)) * D);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t row = at + (uint32_t)((64 * (i / 4) + 4 * (i % 4)) * D);
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(page + (row + (uint32_t)(64 * c + 16 * g)));
#pragma unroll
        for (int e = 0; e < 4; ++e) k[i][4 * c + e] = w[e];
      }
      if constexpr (D % 64 != 0) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(page + (row + (uint32_t)(D / 64 * 64 + 8 * g)));
        k[i][D / 16 - 2] = w[0];
        k[i][D / 16 - 1] = w[1];
      }
    }
  }
};
template <int D>
struct ValuePage {
  u32x4 v[D / 16][2];
  __device__ __forceinline__ void load(const uint8_t* page, int lane) {
    const uint32_t at = (uint32_t)((lane & 15) * kBlock + 16 * (lane >> 4));
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb)
#pragma unroll
      for (int half = 0; half < 2; ++half)
        v[mb][half] = *reinterpret_cast<const u32x4*>(page + (at + (uint32_t)(16 * mb * kBlock + 64 * half)));
  }
};

// The first dim of the 8 that lane group g holds of 32-wide slice m of q and K.
template <int D>
__device__ __forceinline__ int slice_dim(int m, int g) {
  return m < D / 64 * 2 ? 64 * (m / 2) + 16 * g + 8 * (m % 2) : D / 64 * 64 + 8 * g;
}

// Workgroups a compute unit: at 16 rows a wave holds 32 KB of codes in flight or in work, their
// results and the queries in 256 registers, at 32 rows in 512.
template <int RB>
constexpr int cache_wgs() { return RB == 1 ? 2 : 1; }

template <int D, int RB>
__global__ __launch_bounds__(kThreadsC, cache_wgs<RB>()) void cache_attn_kernel(const CacheAttnArgs a) {
  constexpr int kRows = 16 * RB, kWaves = kThreadsC / 64, kMb = D / 16, kSl = D / 32;
  __shared__ float s_o[kWaves][kRows][D + 4];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 15, g = lane >> 4;
  const int w = blockIdx.x, row0 = blockIdx.y * kRows, rows = a.G * a.N;

  // Short tables: a workgroup per segment, and nothing to join (a.whole).
  const Line line(a, !a.whole);
  int lo = 0, hi = INT32_MAX, seg0 = 0, entry, head, len, pages;  // seg0: the line's place where the segment starts
  if (a.whole) {
    entry = scalar_div(w, line.per);
    head = w - entry * line.per;
    len = __builtin_amdgcn_readfirstlane(cache_len(a, entry));
    pages = pages_of(len);
  } else {
    lo = line.start(w);
    hi = line.start(w + 1);
    if (lo >= hi) return;
    entry = line.entry_of(a, lo, seg0);
    len = __builtin_amdgcn_readfirstlane(cache_len(a, entry));
    pages = pages_of(len);
    head = scalar_div(lo - seg0, extent_of(pages));
    seg0 += head * extent_of(pages);
  }

  int at = lo;
  auto advance = [&]() {  // to the next segment with pages; false past the worker's part
    if (a.whole) return false;
    at = seg0 + kSegment + pages;
    if (at >= hi) return false;
    seg0 = at;
    if (++head == line.per) {
      head = 0;
      pages = 0;
      while (pages == 0 && ++entry < line.entries) {
        len = __builtin_amdgcn_readfirstlane(cache_len(a, entry));
        pages = pages_of(len);
      }
    }
    return true;
  };
  do {
    const int b = a.per_head ? scalar_div(entry, a.Hkv) : entry, h = a.per_head ? entry - b * a.Hkv : head;
    const int p0 = max(0, at - seg0 - kSegment), p1 = min(pages, hi - seg0 - kSegment);
    const ScalarInts table = (ScalarInts)(a.table + (size_t)entry * a.max_pages);
    const ScalarFloats k_scales = (ScalarFloats)a.k_scales, v_scales = (ScalarFloats)a.v_scales;
    const size_t q_row = ((size_t)b * a.H + (size_t)h * a.G) * a.N;  // rows of the group lie together

    if (p1 <= p0 && !a.whole) continue;  // (alone, a segment without tokens gets its zeros)
    // Pages p0 + wave, + 4, ... up to p1. A page that is none is passed over: its tokens are not read.
    auto page_of = [&](int p) {
      if (p >= p1) return -1;
      const int x = table[p];
      return x < a.n_pages ? x : -1;
    };
    auto base_of = [&](const uint8_t* pages_at, int page) { return pages_at + ((size_t)page * a.Hkv + h) * kBlock * D; };
    int end[RB];  // tokens this lane's row attends to
    f32x4 o[RB][kMb];
    float m_ref[RB], l_run[RB];
    // All of it; `apart`: NaN codes among the last tokens, which some rows do not see, apart.
    auto attend = [&](auto apart) {
      int p = p0 + wave;
      int page = page_of(p);
      KeyPage<D> kt;
      ValuePage<D> vt;
      if (page >= 0) {
        kt.load(base_of(a.k_pages, page), lane);
        vt.load(base_of(a.v_pages, page), lane);
      }

      bf16x8 qf[RB][kSl];
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
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        m_ref[rb] = kNoRef;
        l_run[rb] = 0.f;
#pragma unroll
        for (int mb = 0; mb < kMb; ++mb) o[rb][mb] = f32x4{0.f, 0.f, 0.f, 0.f};
      }

      // The next page's K loads go out as soon as this one's K is used, its V loads when V is: both
      // have a page's time to arrive, in one set of registers.
      for (; p < p1; p += kWaves) {
        const int next = page_of(p + kWaves);
        const int tok0 = p * kBlock;
        f32x4 s[RB][8];
        float ks = 0.f, vs = 0.f;
        if (page >= 0) {
          ks = k_scales[(size_t)page * a.Hkv + h];
          vs = v_scales[(size_t)page * a.Hkv + h];
          // Fences keep the codes of later slices from being widened early (twice the registers).
#pragma unroll
          for (int m = 0; m < kSl; ++m)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
              for (int i = 4 * half; i < 4 * half + 4; ++i) {
                const bf16x8 kf = widen8(kt.k[i][2 * m], kt.k[i][2 * m + 1]);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                  s[rb][i] = mfma16(kf, qf[rb][m], m == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[rb][i]);
              }
              __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (next >= 0) kt.load(base_of(a.k_pages, next), lane);
        __builtin_amdgcn_sched_barrier(0);
        if (page >= 0) {
          const float c = a.c * ks;
          bf16x8 pf[RB][4];
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[rb][i] *= c;
            if (tok0 + kBlock > len - (a.N - 1)) {
#pragma unroll
              for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (tok0 + 64 * (i / 4) + 16 * g + 4 * (i % 4) + j >= end[rb]) s[rb][i][j] = -INFINITY;
            }
            float mx = s[rb][0][0];
#pragma unroll
            for (int i = 0; i < 8; ++i)
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
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float x = fast_exp2(s[rb][i][j] - m_ref[rb]);
                sum += x;
                pf[rb][i / 2][4 * (i % 2) + j] = (__bf16)(x * vs);
              }
            l_run[rb] += sum;
          }
          if (tok0 + kBlock > len) {  // codes behind the last token may be NaN: clear them in V
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int left = len - (tok0 + 64 * half + 16 * g + 4 * e);
#pragma unroll
                for (int mb = 0; mb < kMb; ++mb) vt.v[mb][half][e] &= bytes_before(left);
              }
          }
          if (decltype(apart)::value && tok0 + kBlock > len - (a.N - 1)) {
            // NaN codes (as ones, 0x38) times the tokens that a row sees: it becomes NaN where that sums to
            // something. Only numbers are added below.
#pragma unroll
            for (int mb = 0; mb < kMb; ++mb) {
              f32x4 sum[RB];
#pragma unroll
              for (int c2 = 0; c2 < 4; ++c2) {
                const int t = tok0 + 64 * (c2 / 2) + 8 * (c2 % 2) + 16 * g;
                uint32_t nan[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  nan[e] = nan_codes(vt.v[mb][c2 / 2][2 * (c2 % 2) + e]);
                  vt.v[mb][c2 / 2][2 * (c2 % 2) + e] &= ~(nan[e] * 0xffu);
                }
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                  const bf16x8 sees = widen8(bytes_before(end[rb] - t) & 0x38383838u, bytes_before(end[rb] - t - 4) & 0x38383838u);
                  sum[rb] = mfma16(widen8(nan[0] * 0x38u, nan[1] * 0x38u), sees, c2 == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sum[rb]);
                }
              }
#pragma unroll
              for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (sum[rb][j] > 0.f) o[rb][mb][j] = __builtin_nanf("");
              __builtin_amdgcn_sched_barrier(0);
            }
          }
#pragma unroll
          for (int mb = 0; mb < kMb; mb += 2) {
#pragma unroll
            for (int c2 = 0; c2 < 4; ++c2)
#pragma unroll
              for (int x = mb; x < mb + 2; ++x) {
                const u32x4 w = vt.v[x][c2 / 2];
                const bf16x8 vf = widen8(w[2 * (c2 % 2)], w[2 * (c2 % 2) + 1]);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) o[rb][x] = mfma16(vf, pf[rb][c2], o[rb][x]);
              }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (next >= 0) vt.load(base_of(a.v_pages, next), lane);
        page = next;
      }
    };
    attend(std::false_type{});
    // The matrix cores add 0 times a NaN to rows that mask its token: where rows see different tokens, a
    // wave that finds a NaN does its pages again with those apart. (In the loop above this took 8%.)
    if (a.N > 1) {
      float worst = 0.f;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int mb = 0; mb < kMb; ++mb)
#pragma unroll
          for (int j = 0; j < 4; ++j) worst += 0.f * o[rb][mb][j];
      if (__builtin_amdgcn_ballot_w64(worst != worst)) attend(std::true_type{});
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
    float* part = a.part + ((size_t)blockIdx.y * 2 * a.workers + slot) * kRows * (D + 4);
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
      const float lse2 = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);  // NaN for a row of NaN
      if (alone) {
        *reinterpret_cast<u32x2*>(a.out + (q_row + row0 + r) * D + d0) =
            __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
        if (a.lse && d0 == 0) a.lse[q_row + row0 + r] = lse2 * 0.69314718055994531f;
      } else {
        float* pr = part + (size_t)r * (D + 4);
        *reinterpret_cast<f32x4*>(pr + d0) = y;
        if (d0 == 0) pr[D] = lse2;
      }
    }
    __syncthreads();
  } while (advance());
}

// Joins the partial results of a segment that several workers share, in the order of its pages;
// a segment without tokens gets its zeros here. A workgroup per segment and 8 rows.
constexpr int kMergeRows = 8;
template <int D, int RB>
__global__ __launch_bounds__(kThreadsC) void cache_merge_kernel(const CacheAttnArgs a) {
  constexpr int kRows = 16 * RB;
  const int b = blockIdx.x / a.Hkv, h = blockIdx.x - b * a.Hkv;
  const int entry = a.per_head ? (int)blockIdx.x : b;
  const int first = blockIdx.y * kMergeRows, rows = min(kMergeRows, a.G * a.N - first);
  const int lane = threadIdx.x & 63;
  const int pages = pages_of(__builtin_amdgcn_readfirstlane(cache_len(a, entry)));
  const Line line(a);
  int before = 0;
  for (int i = lane; i < entry; i += 64) before += extent_of(pages_of(cache_len(a, i)));
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) before += __shfl_xor(before, s);
  const int s0 = __builtin_amdgcn_readfirstlane(before) * line.per + (a.per_head ? 0 : h * extent_of(pages));
  int w0 = 0, w1 = -1;
  if (pages > 0) {
    w0 = line.worker(s0 + kSegment);
    w1 = line.worker(s0 + kSegment + pages - 1);
    if (w0 == w1) return;  // that worker wrote the rows
  }
  const size_t q_row = ((size_t)b * a.H + (size_t)h * a.G) * a.N + first;
  // Worker w's part of the segment: its first one (slot 2 w), or w0's second where that began before.
  const int early = w1 >= w0 && line.start(w0) < s0 ? 1 : 0;
  const float* parts = a.part + (size_t)(first / kRows) * 2 * a.workers * kRows * (D + 4) + (size_t)(first % kRows) * (D + 4);
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreadsC) {
    const int r = i / (D / 4), d0 = 4 * (i % (D / 4));
    const float* pr = parts + (size_t)r * (D + 4);
    const size_t step = (size_t)2 * kRows * (D + 4);
    float m = -INFINITY, l = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int w = w0; w <= w1; ++w) {
      const float* pw = pr + w * step + (w == w0 ? early * (step / 2) : 0);
      const f32x4 u = *reinterpret_cast<const f32x4*>(pw + d0);
      const float part = pw[D], m_new = fmaxf(m, part);
      const float f = part == -INFINITY ? 0.f : fast_exp2(part - m_new);  // a NaN stays one
      const float keep = m == -INFINITY ? 0.f : fast_exp2(m - m_new);
      l = l * keep + f;
      y = y * keep + f * u;
      m = m_new;
    }
    if (l > 0.f) y *= 1.f / l;
    *reinterpret_cast<u32x2*>(a.out + (q_row + r) * D + d0) =
        __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
    if (a.lse && d0 == 0)
      a.lse[q_row + r] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
  }
}

template <int D, int RB>
hipError_t cache_attn_rows(const CacheAttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.workers, (unsigned)a.row_blocks);
  const dim3 segs((unsigned)(a.B * a.Hkv), (unsigned)((a.G * a.N + kMergeRows - 1) / kMergeRows));
  cache_attn_kernel<D, RB><<<grid, kThreadsC, 0, s>>>(a);
  if (!a.whole) cache_merge_kernel<D, RB><<<segs, kThreadsC, 0, s>>>(a);
  return hipGetLastError();
}
template <int D>
hipError_t cache_attn_for(const CacheAttnArgs& a, hipStream_t s) {
  return cache_rows_per_pass(a.G * a.N) == 16 ? cache_attn_rows<D, 1>(a, s) : cache_attn_rows<D, 2>(a, s);
}

}  // namespace

int cache_rows_per_pass(int rows) { return rows <= 16 ? 16 : 32; }

hipError_t launch_cache_write(const CacheWriteArgs& a, hipStream_t stream) {
  // The pages that N tokens can touch, of a table's.
  const int64_t pages = std::min<int64_t>((kBlock - 1 + (int64_t)a.N + kBlock - 1) / kBlock, a.max_pages);
  const dim3 grid((unsigned)pages, (unsigned)(a.B * a.Hkv), 2);
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
