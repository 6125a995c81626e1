// gfx950 (MI355X, CDNA4) kernels of the 4-bit cache: writing it, reading it back, attention over it.
//
// Formats. A page holds 128 tokens of every key head, K and V alike: e2m1 codes [token][d / 2] (two values a byte, the
// even one low) and for every 32 values of a token the exponent of a power of two, [d / 32][token], biased by 127: the
// formats that v_cvt_scalef32_pk_bf16_fp4 takes as they lie, a byte shifted to a float's exponent being the scale.
// Conversions are exact that way (the codes have 2 significant bits), and the other way round to nearest, ties to
// the even code, 6 for what is larger. A token's scales are its own: writing it touches no other one.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <stdint.h>

#include "block_launch.h"
#include "cache_line.h"
#include "tile_common.h"

namespace ta {
namespace {

constexpr int kGroup = 32;  // values that share a scale: four lanes of 8
constexpr int kMinExp4 = -100, kMaxExp4 = 125;
constexpr uint32_t kNanScale = 255;

// ---------------------------------------------------------------------------------------------
// write and read: a token's row of a head takes d / 8 lanes, 8 values (4 bytes of codes) a lane.

template <int D>
struct TokenLanes {
  static constexpr int lanes = D / 8, tokens = 64 / lanes;  // (d = 96: 5 tokens in 60 lanes)
  static constexpr int per_pass = kThreadsC / 64 * tokens;
  static_assert(per_pass == cache4_tokens(D), "tokens of a workgroup");
};

template <int CTRL>
__device__ __forceinline__ uint32_t max_from(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}

// bf16 halves of a word that are infinities or NaN, as a mask of the halves.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// The biased exponent of a group's scale: the least e in [kMinExp4, kMaxExp4] with the largest magnitude at most
// 7 * 2^e. `most`: that magnitude's bf16 bits; it is 1.m * 2^x, and 7 = 1.75 * 2^2.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
  const int x = (int)(most >> 7) - 127;
  const int e = (most & 0x7fu) <= 0x60u ? x - 2 : x - 1;
  return (uint32_t)(min(max(most == 0 ? kMinExp4 : e, kMinExp4), kMaxExp4) + 127);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// (A bit cast of a vector's element takes the first one: elements go through a copy.)
__device__ __forceinline__ bf16x2 as_bf16x2(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }
__device__ __forceinline__ uint32_t encode8(u32x4 w, float scale) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_bf16x2(w[0]), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_bf16x2(w[1]), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_bf16x2(w[2]), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, as_bf16x2(w[3]), scale, 3);
}
__device__ __forceinline__ u32x4 decode8(uint32_t c, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3))};
}

// The page of a position, -1 if it is none.
__device__ __forceinline__ int page_at(const int32_t* table, int max_pages, int n_pages, int64_t pos) {
  const int64_t slot = pos / kBlock;
  if (slot >= max_pages) return -1;
  const int page = table[slot];
  return page < n_pages ? page : -1;
}

// Results go past the caches where all of them together would not stay there for whoever reads them (kStaysInCache): 245 MB of
// read values 50 us so, 63 into the caches, and their reader 77 and 73 us; 31 MB 9.2 and 10.1, and 9.5 and 7.9. (A template: where
// one kernel has both stores, the compiler makes one of them.)
template <bool PAST>
__device__ __forceinline__ void store16(uint16_t* p, u32x4 x) {
  if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = x;
}

// Bound by the bytes: three prompts of 8191 tokens, 8 heads of 96, with the held values 31 us for 171 MB (5.5 TB/s; a large
// copy 5.1); one token of 32 sequences 4.2 us, a chain of loads: length, table, then the stores. A token a lane:
// two, four and eight, read together, took 33, 37 and 75 us.
// K and V of a token in the same lanes: a token that holds anything but finite numbers is marked in K. Scales, bytes
// that lie token by token, are gathered in LDS and leave for all tokens of the workgroup (38 us without).
template <int D, bool PAST>
__global__ __launch_bounds__(kThreadsC) void cache4_write_kernel(const Cache4WriteArgs a) {
  using Lanes = TokenLanes<D>;
  constexpr int kTokens = Lanes::per_pass, kGroups = D / kGroup;
  __shared__ uint8_t s_scale[2 * kGroups * kTokens];  // [K, V][group][token]
  __shared__ int s_page[kTokens];
  const int b = blockIdx.y / a.Hkv, h = blockIdx.y - b * a.Hkv;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sub = lane / Lanes::lanes, l = lane - sub * Lanes::lanes;
  const int64_t len = max(a.lens[b], 0);
  const int n = a.n_new ? min(max(a.n_new[b], 0), a.N) : a.N;
  const int32_t* table = a.table + (size_t)b * a.max_pages;
  const int64_t first = (int64_t)blockIdx.x * kTokens;  // of the workgroup's tokens
  if (sub < Lanes::tokens) {
    const int in_wg = wave * Lanes::tokens + sub;
    const int64_t t = first + in_wg;
    const size_t at = (((size_t)b * a.Hkv + h) * a.N + t) * D + 8 * l;
    u32x4 k = {0u, 0u, 0u, 0u}, v = k;
    int page = -1;
    if (t < n) {
      k = load16(a.k + at);
      v = load16(a.v + at);
      page = page_at(table, a.max_pages, a.n_pages, len + t);
    }
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= not_finite(k[e]) | not_finite(v[e]);
    bool marked = false;
    if (const uint64_t any = __builtin_amdgcn_ballot_w64(bad != 0)) {
      marked = (any >> (sub * Lanes::lanes) & ((1ull << Lanes::lanes) - 1)) != 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        k[e] &= ~not_finite(k[e]);
        v[e] &= ~not_finite(v[e]);
      }
    }
    uint32_t most_k = 0, most_v = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      most_k = max(most_k, max(k[e] & 0x7fffu, k[e] >> 16 & 0x7fffu));
      most_v = max(most_v, max(v[e] & 0x7fffu, v[e] >> 16 & 0x7fffu));
    }
    most_k = max_from<0x4e>(max_from<0xb1>(most_k));  // of four lanes
    most_v = max_from<0x4e>(max_from<0xb1>(most_v));
    uint32_t scale_k = scale_byte(most_k);
    const uint32_t scale_v = scale_byte(most_v);
    const uint32_t code_k = encode8(k, scale_of(scale_k)), code_v = encode8(v, scale_of(scale_v));
    if (marked) scale_k = kNanScale;
    if (l % 4 == 0) {
      s_scale[l / 4 * kTokens + in_wg] = (uint8_t)scale_k;
      s_scale[(kGroups + l / 4) * kTokens + in_wg] = (uint8_t)scale_v;
    }
    if (l == 0) s_page[in_wg] = page;
    if (page >= 0) {
      const size_t code = (((size_t)page * a.Hkv + h) * kBlock + (int)((len + t) % kBlock)) * (D / 2) + 4 * l;
      *reinterpret_cast<uint32_t*>(a.k_pages + code) = code_k;
      *reinterpret_cast<uint32_t*>(a.v_pages + code) = code_v;
    }
    if (t < a.N) {
      const u32x4 none = {0u, 0u, 0u, 0u};
      if (a.k_held) store16<PAST>(a.k_held + at, page < 0 ? none : decode8(code_k, scale_of(scale_k)));
      if (a.v_held) store16<PAST>(a.v_held + at, page < 0 ? none : decode8(code_v, scale_of(scale_v)));
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * kGroups * kTokens; i += kThreadsC) {
    const int in_wg = i % kTokens, row = i / kTokens, page = s_page[in_wg];
    if (page < 0) continue;
    uint8_t* scales = row < kGroups ? a.k_scales : a.v_scales;
    scales[(((size_t)page * a.Hkv + h) * kGroups + row % kGroups) * kBlock + (int)((len + first + in_wg) % kBlock)] =
        s_scale[i];
  }
}

// Bound by the bytes that it writes: 2 sequences of 30001 tokens, 8 heads of 128, 45 us for 300 MB (6.6 TB/s); two and four
// tokens a lane 46 and 49.
template <int D, bool PAST>
__global__ __launch_bounds__(kThreadsC) void cache4_read_kernel(const Cache4ReadArgs a) {
  using Lanes = TokenLanes<D>;
  const int b = blockIdx.y / a.Hkv, h = blockIdx.y - b * a.Hkv;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sub = lane / Lanes::lanes, l = lane - sub * Lanes::lanes;
  const int64_t t = (int64_t)blockIdx.x * Lanes::per_pass + wave * Lanes::tokens + sub, pos = a.first + t;
  if (sub >= Lanes::tokens || t >= a.N) return;
  uint32_t k = 0, v = 0;
  float ks = 1.f, vs = 1.f;
  if (pos < a.lens[b]) {
    const int page = page_at(a.table + (size_t)b * a.max_pages, a.max_pages, a.n_pages, pos);
    if (page >= 0) {
      const int at = (int)(pos % kBlock);
      const size_t ph = (size_t)page * a.Hkv + h;
      const size_t code = (ph * kBlock + at) * (D / 2) + 4 * l, scale = (ph * (D / kGroup) + l / 4) * kBlock + at;
      k = *reinterpret_cast<const uint32_t*>(a.k_pages + code);
      v = *reinterpret_cast<const uint32_t*>(a.v_pages + code);
      ks = scale_of(a.k_scales[scale]);
      vs = scale_of(a.v_scales[scale]);
    }
  }
  const size_t to = (((size_t)b * a.Hkv + h) * a.N + t) * D + 8 * l;
  if (a.k_out) store16<PAST>(a.k_out + to, decode8(k, ks));
  if (a.v_out) store16<PAST>(a.v_out + to, decode8(v, vs));
}

// ---------------------------------------------------------------------------------------------
// attention
//
// A wave takes a page at a time, its codes from memory straight into registers, one page ahead, as operands of
// v_mfma_f32_16x16x32_bf16 (A: lane l holds row l % 16 and the k indices 8 (l / 16) .. + 7; B the same with
// columns; C: column l % 16, rows 4 (l / 16) + j). With n = l % 16 and g = l / 16:
//   S^T = K Q^T. Row n of instruction group i (of 8) is token 8 n + i. The matrix instruction adds over k in any
//   order, so lane group g holds the d / 4 values from g d / 4 on of its token, one load, and q is laid out alike. The
//   scores come out as: lane group g holds tokens 32 g .. 32 g + 31, s[i][j] being token 32 g + 8 j + i,
//   which is the P^T operand of
//   O^T += V^T P^T, step j: its V operand are, of tokens 32 g + 8 j .. + 7, the values of one channel. A lane reads of
//   each of those tokens 4 bytes (2 at d = 64), 8 channels beside each other (4), widens them with the token's scale and
//   swaps halves of words so that words hold two tokens of one channel: the operands of 8 (4) instructions, row n
//   of instruction t being channel 8 n + t (4 n + t).
// P is rounded to bf16 for its product, its sum is not: off by up to 2^-8 of p |v|, below the result's own rounding, and all that the
// results have beside that. In two bf16 parts, with twice the instructions, they come within 1e-6 of fp32 weights' (4e-4 so, of their mean
// magnitude), but 24 sequences of up to 100000 tokens take 125 us for 118, 512 tokens over 32768 (below) 377 for 292.
// So neither K nor V is kept transposed, no scale leaves its token, and nothing goes through LDS. K codes become bf16 exactly,
// scales among it, and so do V's.

// T tokens, all of a page or half of it (above: T = 128; with 64 tokens, row n of instruction group i
// is token 4 n + i, and a lane group has 16 tokens and two steps).
template <int D, int T>
struct Key4 {
  static constexpr int kW = D / 32;  // words of K codes a lane holds of a token, and 8-value slices of them
  static constexpr int kTokens = T / 16;
  uint32_t k[kTokens][kW];
  u32x2 lo, hi;  // scales of the tokens: of the lane's first group of 32 values, and of its last (d = 96)
  __device__ __forceinline__ static u32x2 bytes(const uint8_t* p) {
    if constexpr (kTokens == 8) return *reinterpret_cast<const u32x2*>(p);
    else return u32x2{*reinterpret_cast<const uint32_t*>(p), 0u};
  }
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int lane) {
    const int n = lane & 15, g = lane >> 4, t0 = kTokens * n;
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      const uint8_t* p = codes + (uint32_t)((t0 + i) * (D / 2) + g * (D / 8));
      if constexpr (D == 128) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) k[i][e] = w[e];
      } else if constexpr (D == 64) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(p);
        k[i][0] = w[0];
        k[i][1] = w[1];
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) k[i][e] = reinterpret_cast<const uint32_t*>(p)[e];
      }
    }
    lo = bytes(scales + (uint32_t)(g * kW / 4 * kBlock + t0));
    if constexpr (D == 96) hi = bytes(scales + (uint32_t)((g * kW + kW - 1) / 4 * kBlock + t0));
  }
  // Scales of slice m (of kW).
  __device__ __forceinline__ u32x2 scales_of(int m, int g) const {
    if constexpr (D != 96) return lo;
    const bool last = (g * kW + m) / 4 != g * kW / 4;
    return last ? hi : lo;
  }
};
template <int D, int T>
struct Value4 {
  static constexpr int kSteps = T / 32;
  uint32_t v[kSteps][8];      // token T / 4 g + 8 c + i
  u32x4 scales[kSteps / 2];   // of the lane group's T / 4 tokens
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* group_scales, int lane) {
    const int n = lane & 15, g = lane >> 4, t0 = T / 4 * g;
    // d = 96: lanes 12 to 15 of a group have no channels and read those of lane 11.
    const int word = D == 128 ? n : D == 96 ? min(n, 11) : n / 2, group = D == 64 ? n / 8 : word / 4;
#pragma unroll
    for (int c = 0; c < kSteps; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[c][i] = *reinterpret_cast<const uint32_t*>(codes + (uint32_t)((t0 + 8 * c + i) * (D / 2) + 4 * word));
#pragma unroll
    for (int x = 0; x < kSteps / 2; ++x)
      scales[x] = *reinterpret_cast<const u32x4*>(group_scales + (uint32_t)(group * kBlock + t0 + 16 * x));
  }
};

// Byte i of two words as a scale.
__device__ __forceinline__ float scale_at(u32x2 w, int i) { return scale_of(w[i / 4] >> (8 * (i % 4)) & 0xffu); }

// Two waves a SIMD unit, of 256 registers a lane: enough for a page at 16 rows and for half of one at 32. 24 sequences of up to
// 100000 tokens, 8 key heads of 128: 117 us with 16 rows (5.1 TB/s), 145 with 32 (174 with a whole page, 350
// registers and one wave a unit); of 96, up to 80000, 32 rows: 107 us, 148 so.
template <int D, int RB, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void cache4_attn_kernel(const Cache4AttnArgs a) {
  constexpr int kRows = 16 * RB, kWaves = WAVES, kSl = D / 32;
  constexpr int kT = RB == 1 ? kBlock : kBlock / 2, kParts = kBlock / kT;  // tokens at a time
  constexpr int kGroups = kT / 16, kSteps = kT / 32;
  constexpr int kCh = D == 64 ? 4 : 8;  // channels of a lane, and O^T instructions of a step
  __shared__ float s_o[kWaves][kRows][D + 4];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 15, g = lane >> 4;
  const int row0 = blockIdx.y * kRows, rows = a.G * a.N;

  CacheWalk<kCache4Segment> walk(a, blockIdx.x);
  if (walk.none()) return;
  do {
    const int len = walk.len;
    const CacheSegment seg = walk.segment(a);
    const int p0 = seg.p0, p1 = seg.p1;
    if (p1 <= p0 && !a.whole) continue;  // (alone, a segment without tokens gets its zeros)
    const ScalarInts table = (ScalarInts)(a.table + (size_t)seg.entry * a.max_pages);
    // Pages p0 + wave, + WAVES, ... up to p1. A page that is none is passed over: its tokens are not read.
    auto page_of = [&](int p) {
      if (p >= p1) return -1;
      const int x = table[p];
      return x < a.n_pages ? x : -1;
    };
    auto load_k = [&](Key4<D, kT>& t, int page, int from) {
      const size_t ph = (size_t)page * a.Hkv + seg.h;
      t.load(a.k_pages + (ph * kBlock + from) * (D / 2), a.k_exps + ph * kBlock * (D / kGroup) + from, lane);
    };
    auto load_v = [&](Value4<D, kT>& t, int page, int from) {
      const size_t ph = (size_t)page * a.Hkv + seg.h;
      t.load(a.v_pages + (ph * kBlock + from) * (D / 2), a.v_exps + ph * kBlock * (D / kGroup) + from, lane);
    };
    int p = p0 + wave;
    int page = page_of(p);
    Key4<D, kT> kt;
    Value4<D, kT> vt;
    if (page >= 0) {
      load_k(kt, page, 0);
      load_v(vt, page, 0);
    }

    int end[RB];  // tokens this lane's row attends to
    bf16x8 qf[RB][kSl];
    f32x4 o[RB][kCh];
    float m_ref[RB], l_run[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = row0 + 16 * rb + n;
      end[rb] = r < rows ? len - (a.N - 1) + r % a.N : 0;
#pragma unroll
      for (int m = 0; m < kSl; ++m) {
        u32x4 x = {0u, 0u, 0u, 0u};
        if (r < rows) x = load16(a.q + (seg.q_row + r) * D + 8 * (g * kSl + m));
        qf[rb][m] = as_bf16x8((x ^ a.q_flip) & a.q_keep);
      }
      m_ref[rb] = kNoRef;
      l_run[rb] = 0.f;
#pragma unroll
      for (int t = 0; t < kCh; ++t) o[rb][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // The next tokens' K loads go out as soon as these ones' K is used, their V loads when V is.
    int part = 0, next = page;  // (the page of the next tokens, the same for the page's second half)
    while (p < p1) {
      const int tok0 = p * kBlock + part * kT;
      if (part == kParts - 1) next = page_of(p + kWaves);
      const int next_from = part == kParts - 1 ? 0 : kT;
      f32x4 s[RB][kGroups];
      if (page >= 0) {
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
#pragma unroll
          for (int m = 0; m < kSl; ++m) {
            const bf16x8 kf = as_bf16x8(decode8(kt.k[i][m], scale_at(kt.scales_of(m, g), i)));
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              s[rb][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rb][m], m == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[rb][i], 0, 0, 0);
          }
          if (i % 2) __builtin_amdgcn_sched_barrier(0);  // keeps later tokens' codes from being widened early
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (next >= 0) load_k(kt, next, next_from);
      __builtin_amdgcn_sched_barrier(0);
      if (page >= 0) {
        bf16x8 pf[RB][kSteps];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          if (tok0 + kT > len - (a.N - 1)) {
#pragma unroll
            for (int i = 0; i < kGroups; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (tok0 + kT / 4 * g + kGroups * j + i >= end[rb]) s[rb][i][j] = -INFINITY;
          }
          float mx = s[rb][0][0];
#pragma unroll
          for (int i = 0; i < kGroups; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) mx = fmaxf(mx, s[rb][i][j]);
          const float m_new = fmaxf(m_ref[rb], group_max(mx) * a.c);
          if (__builtin_amdgcn_ballot_w64(m_new > m_ref[rb])) {
            const float alpha = fast_exp2(m_ref[rb] - m_new);
            l_run[rb] *= alpha;
#pragma unroll
            for (int t = 0; t < kCh; ++t) o[rb][t] *= alpha;
            m_ref[rb] = m_new;
          }
          float c = a.c;
          if (__builtin_expect(__builtin_amdgcn_ballot_w64(is_far(m_ref[rb])) != 0, 0)) {  // (rows that are not keep theirs)
            const bool far = is_far(m_ref[rb]);
#pragma unroll
            for (int i = 0; i < kGroups; ++i) s[rb][i] *= far ? c : 1.f;
            c = far ? 1.f : c;
          }
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < kGroups; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x = fast_exp2(fmaf(s[rb][i][j], c, -m_ref[rb]));
              sum += x;
              pf[rb][(kGroups * j + i) / 8][(kGroups * j + i) % 8] = (__bf16)x;
            }
          l_run[rb] += sum;
        }
        if (tok0 + kT > len) {  // scales behind the last token may be anything: those of V become 2^-127
#pragma unroll
          for (int x = 0; x < kSteps / 2; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) vt.scales[x][e] &= bytes_before(len - (tok0 + kT / 4 * g + 16 * x + 4 * e));
        }
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
          // vf[t]: of channel t of the lane, the step's 8 tokens.
          u32x4 vf[kCh];
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const u32x2 sc = {vt.scales[c / 2][2 * (c % 2)], vt.scales[c / 2][2 * (c % 2) + 1]};
            const float s0 = scale_at(sc, i), s1 = scale_at(sc, i + 1);
            uint32_t w0 = vt.v[c][i], w1 = vt.v[c][i + 1];
            if constexpr (D == 64) {
              w0 >>= 16 * (n & 1);
              w1 >>= 16 * (n & 1);
            }
            const u32x4 x0 = decode8(w0, s0), x1 = decode8(w1, s1);
#pragma unroll
            for (int y = 0; y < kCh / 2; ++y) {
              vf[2 * y][i / 2] = __builtin_amdgcn_perm(x1[y], x0[y], 0x05040100u);
              vf[2 * y + 1][i / 2] = __builtin_amdgcn_perm(x1[y], x0[y], 0x07060302u);
            }
          }
#pragma unroll
          for (int t = 0; t < kCh; ++t)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              o[rb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[t]), pf[rb][c], o[rb][t], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (next >= 0) load_v(vt, next, next_from);
      page = next;
      if (part == kParts - 1) {
        p += kWaves;
        part = 0;
      } else {
        ++part;
      }
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
      for (int j = 0; j < 4; ++j) {
        const int ch = kCh * (4 * g + j);
        if (ch >= D) continue;
#pragma unroll
        for (int t = 0; t < kCh; t += 4)
          *reinterpret_cast<f32x4*>(&s_o[wave][16 * rb + n][ch + t]) =
              f32x4{o[rb][t][j], o[rb][t + 1][j], o[rb][t + 2][j], o[rb][t + 3][j]};
      }
    }
    __syncthreads();
    join_waves<D>(a, s_o, s_m, s_l, seg.q_row, row0, rows, seg.alone, seg.slot);
    __syncthreads();
  } while (walk.advance(a));
}

// Many rows. Above, every 32 rows of a key head widen every page again. Here a workgroup of eight waves has four sets of
// 16 RB rows, each with a wave for the first half of a page's tokens and one for the second, which join at the end: a page's codes are
// widened once, K by four waves and V by the other four, into LDS, where the matrix operands of all rows come from.
// While a page is multiplied the next one is widened into the other half of the LDS, and the one behind it is on its way.
// Bound by the vector work beside the products (exponentials, widening): one sequence of 32768, 32 heads on 8 of 128, the last 2048 tokens
// 1107 us (993 TFLOP/s), 512 workgroups of four waves that had a page's tokens to themselves 1166. 128 rows take 2.3 us a
// page at d = 128, 2.6 at 96 (of which 2.0 for scores, exponentials and products, 0.5 for widening). Waves of K widening before their products and waves of V behind them: 1261; two sets of 48 rows, four
// waves each, for 96 rows: 36.3 us for 32.5, the joins of four waves cost more than the even rows give.
//   K: row 16 i + n of the tile is the token that row n of instruction group i computes, 32 (i / 2) + 8 (n / 4) + 4 (i % 2) + n % 4,
//   so that the scores of groups 2 c and 2 c + 1 are, in lane group g, tokens 32 c + 8 g .. + 7: P^T of step c. The 16-byte pieces
//   of a row lie at places exchanged by the row's number (d = 64: in order, rows 16 bytes longer than their values), which puts
//   16 rows' pieces on different banks (2048 tokens over 32768: 1107 us, 1124 with longer rows).
//   V^T: a row of 128 tokens for each channel, its 16-byte pieces of 8 tokens at places exchanged by the channel's
//   number (key): both the writes (16 channels' words of the same 8 tokens) and the reads (row n of instruction t: channel 8 n + t,
//   4 n + t at d = 64) fall on different banks.
constexpr int kThreadsMany = 512;
template <int D, int RB>
__global__ __launch_bounds__(kThreadsMany, 2) void cache4_rows_kernel(const Cache4AttnArgs a) {
  constexpr int kSets = 4, kRows = 16 * RB * kSets, kSl = D / 32;
  constexpr int kParts = 2, kT = kBlock / kParts;  // of a page, and their tokens
  constexpr int kGroups = kT / 16, kSteps = kT / 32;
  constexpr int kCh = D == 64 ? 4 : 8;
  constexpr int kPitch = D == 64 ? 72 : 128;          // of a K row, in values
  constexpr int kHalf = kThreadsMany / 2;             // threads that widen K, and V
  constexpr int kKUnits = kBlock * (D / kGroup);      // 32 values of a token
  constexpr int kKPer = (kKUnits + kHalf - 1) / kHalf;
  constexpr int kWords = D / 8;                       // of a token's codes
  constexpr int kVUnits = kBlock / 8 * kWords;        // a word of 8 tokens
  static_assert(kKPer <= 2 && kVUnits <= kHalf, "codes a thread widens");
  constexpr int kPage = kBlock * kPitch + D * kBlock;  // a widened page, in values
  constexpr int kLanes = D == 96 ? 48 : 64;            // that hold channels
  constexpr int kState = kLanes * RB * (kCh + 1);      // 16-byte pieces of a wave's state
  static_assert(kSets * kState * 16 <= 2 * kPage * 2, "states take the pages' place");
  __shared__ __attribute__((aligned(16))) uint16_t s_page[2 * kPage];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 15, g = lane >> 4;
  const int set = wave % kSets, part = wave / kSets;  // rows, and tokens kT part .. of a page
  const int rows = a.G * a.N, row0 = blockIdx.y * kRows + 16 * RB * set;
  const bool works = row0 < rows;
  const bool for_k = wave < 4;  // what it widens
  auto k_key = [](int row) { return D == 64 ? 0 : row & 15; };  // places of a K row's pieces
  const int unit = tid % kHalf;
  const int v_word = unit % kWords, v_part = unit / kWords;  // tokens 8 v_part .. + 7

  CacheWalk<kCache4Segment> walk(a, blockIdx.x);
  if (walk.none()) return;
  do {
    const int len = walk.len;
    const CacheSegment seg = walk.segment(a);
    const int p0 = seg.p0, p1 = seg.p1;
    if (p1 <= p0 && !a.whole) continue;  // (alone, a segment without tokens gets its zeros)
    const ScalarInts table = (ScalarInts)(a.table + (size_t)seg.entry * a.max_pages);
    // The next page from p on that is one; its number in `page`.
    int page = -1;
    auto seek = [&](int p) {
      for (; p < p1; ++p) {
        page = table[p];
        if (page >= 0 && page < a.n_pages) break;
      }
      return p;
    };
    u32x4 cw[2];     // K: 16 bytes of codes; V: words of 8 tokens
    uint32_t sc[2];  // their scales
    // (Every thread loads, the last unit again where there are fewer: without a branch the loads stay on their way.)
    auto load = [&]() {
      const size_t ph = (size_t)page * a.Hkv + seg.h;
      if (for_k) {
        const uint8_t* k = a.k_pages + ph * kBlock * (D / 2);
        const uint8_t* ke = a.k_exps + ph * kBlock * (D / kGroup);
#pragma unroll
        for (int i = 0; i < kKPer; ++i) {
          const int u = min(unit + kHalf * i, kKUnits - 1), t = u / (D / kGroup), grp = u % (D / kGroup);
          cw[i] = *reinterpret_cast<const u32x4*>(k + (uint32_t)(t * (D / 2) + 16 * grp));
          sc[i] = ke[(uint32_t)(grp * kBlock + t)];
        }
      } else {
        const uint8_t* v = a.v_pages + ph * kBlock * (D / 2);
        const uint8_t* ve = a.v_exps + ph * kBlock * (D / kGroup);
        const int u = min(unit, kVUnits - 1), word = u % kWords, part = u / kWords;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          cw[i / 4][i % 4] = *reinterpret_cast<const uint32_t*>(v + (uint32_t)((8 * part + i) * (D / 2) + 4 * word));
        const u32x2 vs = *reinterpret_cast<const u32x2*>(ve + (uint32_t)(word / 4 * kBlock + 8 * part));
        sc[0] = vs[0];
        sc[1] = vs[1];
      }
    };
    auto widen = [&](uint16_t* s_k, int p) {
      if (for_k) {
#pragma unroll
        for (int i = 0; i < kKPer; ++i) {
          const int u = unit + kHalf * i, t = u / (D / kGroup), grp = u % (D / kGroup);
          if (u < kKUnits) {
            const int row = (t & ~31) + 16 * (t >> 2 & 1) + 4 * (t >> 3 & 3) + (t & 3);
            const float f = scale_of(sc[i]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<u32x4*>(s_k + row * kPitch + 8 * ((4 * grp + e) ^ k_key(row))) = decode8(cw[i][e], f);
          }
        }
      } else if (unit < kVUnits) {
        uint16_t* s_v = s_k + kBlock * kPitch;
        // Scales behind the last token may be anything: theirs become 2^-127.
        const int left = len - (p * kBlock + 8 * v_part);
        const u32x2 vs = {sc[0] & bytes_before(left), sc[1] & bytes_before(left - 4)};
        u32x4 x[8];  // of the word's 8 channels
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const u32x4 x0 = decode8(cw[i / 4][i % 4], scale_at(vs, i));
          const u32x4 x1 = decode8(cw[i / 4][i % 4 + 1], scale_at(vs, i + 1));
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            x[2 * y][i / 2] = __builtin_amdgcn_perm(x1[y], x0[y], 0x05040100u);
            x[2 * y + 1][i / 2] = __builtin_amdgcn_perm(x1[y], x0[y], 0x07060302u);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int ch = 8 * v_word + e, key = ch / kCh;
          *reinterpret_cast<u32x4*>(s_v + ch * kBlock + 8 * (v_part ^ key)) = x[e];
        }
      }
    };

    int p = seek(p0);
    if (p < p1) load();
    int end[RB];  // tokens this lane's row attends to
    bf16x8 qf[RB][kSl];
    f32x4 o[RB][kCh];
    float m_ref[RB], l_run[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = row0 + 16 * rb + n;
      end[rb] = r < rows ? len - (a.N - 1) + r % a.N : 0;
#pragma unroll
      for (int m = 0; m < kSl; ++m) {
        u32x4 x = {0u, 0u, 0u, 0u};
        if (r < rows) x = load16(a.q + (seg.q_row + r) * D + 32 * m + 8 * g);
        qf[rb][m] = as_bf16x8((x ^ a.q_flip) & a.q_keep);
      }
      m_ref[rb] = kNoRef;
      l_run[rb] = 0.f;
#pragma unroll
      for (int t = 0; t < kCh; ++t) o[rb][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    int now = p;  // the page that is multiplied, the next one being widened and p the one on its way
    uint16_t* s_now = s_page;
    uint16_t* s_next = s_page + kPage;
    if (now < p1) {
      widen(s_now, now);
      p = seek(now + 1);
      if (p < p1) load();
      __syncthreads();
    }
    while (now < p1) {
      const int tok0 = now * kBlock + kT * part;
      now = p;
      if (now < p1) {
        widen(s_next, now);
        p = seek(now + 1);
        if (p < p1) load();
      }
      if (works) {
        const uint16_t* s_k = s_now + kT * part * kPitch;
        const uint16_t* s_v = s_now + kBlock * kPitch;
        f32x4 s[RB][kGroups];
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
#pragma unroll
          for (int m = 0; m < kSl; ++m) {
            const bf16x8 kf = as_bf16x8(*reinterpret_cast<const u32x4*>(s_k + (16 * i + n) * kPitch + 8 * ((4 * m + g) ^ k_key(n))));
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              s[rb][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rb][m], m == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[rb][i], 0, 0, 0);
          }
        // Four K pieces are on their way from LDS while RB products use one (one sequence of 32768, 8 heads, 512 rows each: 315 us,
        // 329 as the compiler orders them, with four waves).
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int x = 0; x < kGroups * kSl - 4; ++x) {
          __builtin_amdgcn_sched_group_barrier(0x008, RB, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4 * RB, 0);
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 pf[RB][kSteps];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          if (tok0 + kT > len - (a.N - 1)) {
#pragma unroll
            for (int i = 0; i < kGroups; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (tok0 + 32 * (i / 2) + 8 * g + 4 * (i % 2) + j >= end[rb]) s[rb][i][j] = -INFINITY;
          }
          float mx = s[rb][0][0];
#pragma unroll
          for (int i = 0; i < kGroups; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) mx = fmaxf(mx, s[rb][i][j]);
          const float m_new = fmaxf(m_ref[rb], group_max(mx) * a.c);
          if (__builtin_amdgcn_ballot_w64(m_new > m_ref[rb])) {
            const float alpha = fast_exp2(m_ref[rb] - m_new);
            l_run[rb] *= alpha;
#pragma unroll
            for (int t = 0; t < kCh; ++t) o[rb][t] *= alpha;
            m_ref[rb] = m_new;
          }
        }
        // (One question for all rows: 512 tokens over 32768, 32 heads on 8, take 2% more with one for each 16 rows, and 3% with
        // rounded products everywhere.)
        float c[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) c[rb] = a.c;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(is_far(m_ref[0]) || is_far(m_ref[RB - 1])) != 0, 0)) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            const bool far = is_far(m_ref[rb]);
#pragma unroll
            for (int i = 0; i < kGroups; ++i) s[rb][i] *= far ? a.c : 1.f;
            c[rb] = far ? 1.f : a.c;
          }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < kGroups; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x = fast_exp2(fmaf(s[rb][i][j], c[rb], -m_ref[rb]));
              sum += x;
              pf[rb][i / 2][4 * (i % 2) + j] = (__bf16)x;
            }
          l_run[rb] += sum;
        }
#pragma unroll
        for (int c = 0; c < kSteps; ++c)
#pragma unroll
          for (int t = 0; t < kCh; ++t) {
            // (d = 96: rows 12 to 15 of an instruction are no channels and read those of rows 0 to 3.)
            const int key = D == 96 && n > 11 ? n - 12 : n;
            const bf16x8 vf = as_bf16x8(*reinterpret_cast<const u32x4*>(s_v + (kCh * key + t) * kBlock + 8 * ((kT / 8 * part + 4 * c + g) ^ key)));
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              o[rb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rb][c], o[rb][t], 0, 0, 0);
          }
      }
      __syncthreads();  // this page is done with, the next one is there
      uint16_t* x = s_now;
      s_now = s_next;
      s_next = x;
    }

    // The states of a set's two waves join, through the pages' place, each lane its own.
    f32x4* state = reinterpret_cast<f32x4*>(s_page) + set * kState;
    if (works && part == 1) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float l = group_sum(l_run[rb]);
        f32x4* to = state + kLanes * rb * (kCh + 1);
        if (g == 0) to[kLanes * kCh + n] = f32x4{m_ref[rb], l, 0.f, 0.f};
        if (lane < kLanes) {
#pragma unroll
          for (int t = 0; t < kCh; ++t) to[kLanes * t + lane] = o[rb][t];
        }
      }
    }
    __syncthreads();
    // A wave's rows are its own: results or partial results straight from its registers.
    if (part == 0 && works) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const f32x4* from = state + kLanes * rb * (kCh + 1);
        const f32x4 other = from[kLanes * kCh + n];
        const float m = fmaxf(m_ref[rb], other[0]);
        float f0 = fast_exp2(m_ref[rb] - m), f1 = fast_exp2(other[0] - m);
        const float l = group_sum(l_run[rb]) * f0 + other[1] * f1;
        const int r = row0 + 16 * rb + n;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        f0 *= inv;
        f1 *= inv;
#pragma unroll
        for (int t = 0; t < kCh; ++t) o[rb][t] = o[rb][t] * f0 + from[kLanes * t + min(lane, kLanes - 1)] * f1;
        // (A row of NaN stays one: its sums are NaN, and so is its quotient's product.)
        const float lse2 = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);
        if (r >= rows) continue;
        float* pr = a.part + (((size_t)blockIdx.y * 2 * a.workers + seg.slot) * kRows + 16 * (RB * set + rb) + n) * (D + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int ch = kCh * (4 * g + j);
          if (ch >= D) continue;
#pragma unroll
          for (int t = 0; t < kCh; t += 4) {
            const f32x4 y = f32x4{o[rb][t][j], o[rb][t + 1][j], o[rb][t + 2][j], o[rb][t + 3][j]};
            if (seg.alone)
              *reinterpret_cast<u32x2*>(a.out + (seg.q_row + r) * D + ch + t) =
                  __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
            else
              *reinterpret_cast<f32x4*>(pr + ch + t) = y;
          }
        }
        if (g == 0) {
          if (!seg.alone) pr[D] = lse2;
          else if (a.lse) a.lse[seg.q_row + r] = lse2 * 0.69314718055994531f;
        }
      }
    }
    __syncthreads();
  } while (walk.advance(a));
}

constexpr int kMergeSlices = 8;
template <int D, int ROWS>
hipError_t cache4_attn_rows(const Cache4AttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.workers, (unsigned)a.row_blocks);
  if constexpr (ROWS > 32) {
    cache4_rows_kernel<D, ROWS / 64><<<grid, kThreadsMany, 0, s>>>(a);
  } else {
    if (ROWS == 16 && a.eight) cache4_attn_kernel<D, 1, 8><<<grid, 512, 0, s>>>(a);
    else cache4_attn_kernel<D, ROWS / 16, 4><<<grid, kThreadsC, 0, s>>>(a);
  }
  if (a.whole) return hipGetLastError();
  const int segments = a.B * a.Hkv, rows = a.G * a.N;
  auto segs = [&](int per) { return dim3((unsigned)segments, (unsigned)((rows + per - 1) / per)); };
  if (a.workers > 4 * segments)
    cache_merge_kernel<D, ROWS / 16, kCache4Segment, kMergeSlices><<<segs(merge_rows<D, kMergeSlices>()), kThreadsC, 0, s>>>(a);
  else
    cache_merge_kernel<D, ROWS / 16, kCache4Segment><<<segs(kMergeRows), kThreadsC, 0, s>>>(a);
  return hipGetLastError();
}
template <int D>
hipError_t cache4_attn_for(const Cache4AttnArgs& a, hipStream_t s) {
  switch (cache4_rows_per_pass(a.G * a.N)) {
    case 16: return cache4_attn_rows<D, 16>(a, s);
    case 32: return cache4_attn_rows<D, 32>(a, s);
    case 64: return cache4_attn_rows<D, 64>(a, s);
    default: return cache4_attn_rows<D, 128>(a, s);
  }
}

template <int D>
dim3 token_grid(int N, int heads) {
  constexpr int per = TokenLanes<D>::per_pass;
  return dim3((unsigned)(((int64_t)N + per - 1) / per), (unsigned)heads);
}

template <int D>
hipError_t write_tokens(const Cache4WriteArgs& a, hipStream_t s) {
  const dim3 grid = token_grid<D>(a.N, a.B * a.Hkv);
  if (a.past) cache4_write_kernel<D, true><<<grid, kThreadsC, 0, s>>>(a);
  else cache4_write_kernel<D, false><<<grid, kThreadsC, 0, s>>>(a);
  return hipGetLastError();
}
template <int D>
hipError_t read_tokens(const Cache4ReadArgs& a, hipStream_t s) {
  const dim3 grid = token_grid<D>(a.N, a.B * a.Hkv);
  if (a.past) cache4_read_kernel<D, true><<<grid, kThreadsC, 0, s>>>(a);
  else cache4_read_kernel<D, false><<<grid, kThreadsC, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

int cache4_rows_per_pass(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }

hipError_t launch_cache4_write(const Cache4WriteArgs& a, hipStream_t s) {
  if (a.d == 64) return write_tokens<64>(a, s);
  return a.d == 96 ? write_tokens<96>(a, s) : write_tokens<128>(a, s);
}

hipError_t launch_cache4_read(const Cache4ReadArgs& a, hipStream_t s) {
  if (a.d == 64) return read_tokens<64>(a, s);
  return a.d == 96 ? read_tokens<96>(a, s) : read_tokens<128>(a, s);
}

hipError_t launch_cache4_attn(const Cache4AttnArgs& a, hipStream_t stream) {
  if (a.d == 64) return cache4_attn_for<64>(a, stream);
  if (a.d == 96) return cache4_attn_for<96>(a, stream);
  return cache4_attn_for<128>(a, stream);
}

}  // namespace ta
