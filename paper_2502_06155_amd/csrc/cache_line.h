// What attention over the 8-bit and the 4-bit cache share: how the pages of all sequences are dealt out to
// workgroups, and how partial results are joined.
#pragma once
#include <hip/hip_runtime.h>

#include <cfloat>
#include <stdint.h>

#include "block_launch.h"
#include "tile_common.h"

namespace ta {
namespace {

constexpr int kThreadsC = 256;

// A quotient of numbers that are the same in every lane, in a scalar register (the division itself runs
// on the vector ALU; left there, it would make every address and branch behind it a lane's own).
__device__ __forceinline__ int scalar_div(int x, int y) {
  return __builtin_amdgcn_readfirstlane((int)((uint32_t)x / (uint32_t)y));
}

// The line of all segments, each SEGMENT + its pages long (below 2^31, checked by the host): what a
// segment's start and end cost a workgroup is about SEGMENT pages' time (8 bits, 32 sequences of 4 to 512
// pages: 208 us with 0, 188 with 3). Segment order: entry i of lens, then (where all heads share an
// entry) the key heads. Worker w takes line / workers, the first line % workers ones one more. Every
// wave finds its place by itself, 64 entries at a time.
using ScalarInts = const __attribute__((address_space(4))) int32_t*;  // read with scalar loads

__device__ __forceinline__ int cache_len(const CacheAttnArgs& a, int i) {
  return (int)min((int64_t)max(a.lens[i], 0), (int64_t)a.max_pages * kBlock);
}
__device__ __forceinline__ int pages_of(int len) { return (int)(((uint32_t)len + kBlock - 1) / kBlock); }
// A segment's length on the line; one without pages has none.
template <int SEGMENT>
__device__ __forceinline__ int extent_of(int pages) { return pages > 0 ? SEGMENT + pages : 0; }

// The sum of a number over the lanes up to one's own: shifts inside 16 lanes, then the rows' last lanes handed on.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_lanes(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int sum_upto(int x) {
  x = add_lanes<0x111, 0xf>(x);  // from the lane 1, 2, 4, 8 before, in a row of 16
  x = add_lanes<0x112, 0xf>(x);
  x = add_lanes<0x114, 0xf>(x);
  x = add_lanes<0x118, 0xf>(x);
  x = add_lanes<0x142, 0xa>(x);  // lane 15 to the row behind it, rows 1 and 3
  return add_lanes<0x143, 0xc>(x);  // lane 31 to rows 2 and 3
}
__device__ __forceinline__ int sum_all(int x) { return __builtin_amdgcn_readlane(sum_upto(x), 63); }

template <int SEGMENT>
struct CacheLine {
  int entries, per;  // entries of lens, segments of an entry
  int total;         // its length
  int each, more;    // every worker's part, workers with one more
  __device__ __forceinline__ CacheLine(const CacheAttnArgs& a, bool measure = true) {
    entries = a.per_head ? a.B * a.Hkv : a.B;
    per = a.per_head ? 1 : a.Hkv;
    total = each = more = 0;
    if (!measure) return;
    int n = 0;
    for (int i = threadIdx.x & 63; i < entries; i += 64) n += extent_of<SEGMENT>(pages_of(cache_len(a, i)));
    total = sum_all(n) * per;
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
      const int own = i0 + lane < entries ? extent_of<SEGMENT>(pages_of(cache_len(a, i0 + lane))) * per : 0;
      const int upto = sum_upto(own);
      const uint64_t past = __builtin_amdgcn_ballot_w64(before + upto > at);
      if (past) {
        const int src = __ffsll((unsigned long long)past) - 1;
        before += __builtin_amdgcn_readlane(upto - own, src);
        return i0 + src;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    return entries;
  }
};

// max and sum over the four lane groups that hold one query row's tokens.
__device__ __forceinline__ float group_max(float x) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);  // groups 0 0 2 2, 1 1 3 3
  return pair_max(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])));
}
__device__ __forceinline__ float group_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The bytes of a word that come before byte `left`.
__device__ __forceinline__ uint32_t bytes_before(int left) {
  return left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
}
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

constexpr float kNoRef = -FLT_MAX;  // a running maximum before the first token (base-2 logits)
// A row's logits are so far from 0 that their products with c have to be rounded as their maximum's was: in the exact difference
// of fma(s, c, -m) the rounding of m, up to 2^-24 of it, would leave the exponent's range from 2^31 on.
__device__ __forceinline__ bool is_far(float m) { return fabsf(m) > 0x1p24f && m > kNoRef; }

// A part of a segment: pages p0 .. p1 - 1 of key head h of an entry of lens, the group's first query row, whether
// that is the whole segment, and the slot of the partial result if it is not.
struct CacheSegment {
  int entry, h, p0, p1;
  size_t q_row;
  bool alone;
  int slot;
};

// The segments that worker w's stretch of the line meets, one after the other. Short tables: a workgroup per
// segment, and nothing to join (a.whole).
template <int SEGMENT>
struct CacheWalk {
  CacheLine<SEGMENT> line;
  int w, lo = 0, hi = INT32_MAX, seg0 = 0, at, entry, head, len, pages;  // seg0: the line's place where the segment starts
  __device__ __forceinline__ CacheWalk(const CacheAttnArgs& a, int worker) : line(a, !a.whole), w(worker) {
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
      head = scalar_div(lo - seg0, extent_of<SEGMENT>(pages));
      seg0 += head * extent_of<SEGMENT>(pages);
    }
    at = lo;
  }
  __device__ __forceinline__ bool none() const { return lo >= hi; }
  __device__ __forceinline__ bool advance(const CacheAttnArgs& a) {  // to the next segment with pages; false past the part
    if (a.whole) return false;
    at = seg0 + SEGMENT + pages;
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
  }
  __device__ __forceinline__ CacheSegment segment(const CacheAttnArgs& a) const {
    CacheSegment s;
    const int b = a.per_head ? scalar_div(entry, a.Hkv) : entry;
    s.entry = entry;
    s.h = a.per_head ? entry - b * a.Hkv : head;
    s.p0 = max(0, at - seg0 - SEGMENT);
    s.p1 = min(pages, hi - seg0 - SEGMENT);
    s.q_row = ((size_t)b * a.H + (size_t)s.h * a.G) * a.N;  // rows of the group lie together
    s.alone = s.p0 == 0 && s.p1 == pages;
    s.slot = 2 * w + (at == lo ? 0 : 1);
    return s;
  }
};

// The waves' states (sums of weighted values, running maxima in base 2, sums of weights) become the
// segment's results, or one of its partial results.
template <int D, int ROWS, int WAVES>
__device__ __forceinline__ void join_waves(const CacheAttnArgs& a, const float (&s_o)[WAVES][ROWS][D + 4],
                                           const float (&s_m)[WAVES][ROWS], const float (&s_l)[WAVES][ROWS],
                                           size_t q_row, int row0, int rows, bool alone, int slot) {
  float* part = a.part + ((size_t)blockIdx.y * 2 * a.workers + slot) * ROWS * (D + 4);
  for (int i = threadIdx.x; i < ROWS * (D / 4); i += 64 * WAVES) {
    const int r = i / (D / 4), d0 = 4 * (i % (D / 4));
    if (row0 + r >= rows) continue;
    float m = s_m[0][r];
#pragma unroll
    for (int x = 1; x < WAVES; ++x) m = fmaxf(m, s_m[x][r]);
    float l = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < WAVES; ++x) {
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
}

// Joins the partial results of a segment that several workers share, in the order of its pages;
// a segment without tokens gets its zeros here. A workgroup per segment and 8 rows; or, where many workers
// share a segment, its threads share a row's parts in SLICES slices (part w is slice w % SLICES'), joined in LDS.
constexpr int kMergeRows = 8;
template <int D, int SLICES>
constexpr int merge_rows() { return SLICES == 1 ? kMergeRows : kThreadsC / (SLICES * (D / 4)); }
template <int D, int RB, int SEGMENT, int SLICES = 1>
__global__ __launch_bounds__(kThreadsC) void cache_merge_kernel(const CacheAttnArgs a) {
  constexpr int kRows = 16 * RB, kPer = merge_rows<D, SLICES>();
  static_assert(kRows % kPer == 0, "a workgroup's rows are of one pass");
  __shared__ float s_y[SLICES > 1 ? SLICES * kPer : 1][D + 4];  // a slice's sum, weight and maximum
  const int b = blockIdx.x / a.Hkv, h = blockIdx.x - b * a.Hkv;
  const int entry = a.per_head ? (int)blockIdx.x : b;
  const int first = blockIdx.y * kPer, rows = min(kPer, a.G * a.N - first);
  const int lane = threadIdx.x & 63;
  const int pages = pages_of(__builtin_amdgcn_readfirstlane(cache_len(a, entry)));
  const CacheLine<SEGMENT> line(a);
  int before = 0;
  for (int i = lane; i < entry; i += 64) before += extent_of<SEGMENT>(pages_of(cache_len(a, i)));
  const int s0 = sum_all(before) * line.per + (a.per_head ? 0 : h * extent_of<SEGMENT>(pages));
  int w0 = 0, w1 = -1;
  if (pages > 0) {
    w0 = line.worker(s0 + SEGMENT);
    w1 = line.worker(s0 + SEGMENT + pages - 1);
    if (w0 == w1) return;  // that worker wrote the rows
  }
  const size_t q_row = ((size_t)b * a.H + (size_t)h * a.G) * a.N + first;
  // Worker w's part of the segment: its first one (slot 2 w), or w0's second where that began before.
  const int early = w1 >= w0 && line.start(w0) < s0 ? 1 : 0;
  const float* parts = a.part + (size_t)(first / kRows) * 2 * a.workers * kRows * (D + 4) + (size_t)(first % kRows) * (D + 4);
  const size_t step = (size_t)2 * kRows * (D + 4);
  // Adds a partial result, of log-sum-exp `part` and with weight `weight` in it, to a running one.
  auto add = [](float part, float weight, f32x4 u, float& m, float& l, f32x4& y) {
    const float m_new = fmaxf(m, part);
    const float f = part == -INFINITY ? 0.f : fast_exp2(part - m_new) * weight;  // a NaN stays one
    const float keep = m == -INFINITY ? 0.f : fast_exp2(m - m_new);
    l = l * keep + f;
    y = y * keep + f * u;
    m = m_new;
  };
  auto write = [&](int r, int d0, float m, float l, f32x4 y) {
    if (l > 0.f) y *= 1.f / l;
    *reinterpret_cast<u32x2*>(a.out + (q_row + r) * D + d0) =
        __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
    if (a.lse && d0 == 0)
      a.lse[q_row + r] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
  };
  const int items = rows * (D / 4) * SLICES;
  for (int i = threadIdx.x; i < items; i += kThreadsC) {
    const int slice = SLICES == 1 ? 0 : i / (D / 4) % SLICES, r = i / (D / 4 * SLICES), d0 = 4 * (i % (D / 4));
    const float* pr = parts + (size_t)r * (D + 4);
    float m = -INFINITY, l = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int w = w0 + slice; w <= w1; w += SLICES) {
      const float* pw = pr + w * step + (w == w0 ? early * (step / 2) : 0);
      add(pw[D], 1.f, *reinterpret_cast<const f32x4*>(pw + d0), m, l, y);
    }
    if constexpr (SLICES == 1) {
      write(r, d0, m, l, y);
    } else {
      float* to = s_y[r * SLICES + slice];
      *reinterpret_cast<f32x4*>(to + d0) = l > 0.f ? y * (1.f / l) : y;  // (a NaN stays one)
      if (d0 == 0) {
        to[D] = l;
        to[D + 1] = m;
      }
    }
  }
  if constexpr (SLICES > 1) {
    __syncthreads();
    for (int i = threadIdx.x; i < rows * (D / 4); i += kThreadsC) {
      const int r = i / (D / 4), d0 = 4 * (i % (D / 4));
      float m = -INFINITY, l = 0.f;
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < SLICES; ++x) {
        const float* from = s_y[r * SLICES + x];
        const float weight = from[D];
        // (A slice of NaN parts alone has no maximum: its weight, NaN, stands for it.)
        const float top = weight == 0.f ? -INFINITY : weight > 0.f ? from[D + 1] : weight;
        add(top, weight, *reinterpret_cast<const f32x4*>(from + d0), m, l, y);
      }
      write(r, d0, m, l, y);
    }
  }
}

}  // namespace
}  // namespace ta
