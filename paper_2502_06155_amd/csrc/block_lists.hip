// gfx950 (MI355X, CDNA4) kernels that choose key blocks: block means and lists.
//
// The mean of a block is summed in 64 bits: bf16 values have 8-bit significands, so a sum of up
// to a few thousand of them is exact unless their magnitudes span more than 2^30, and the one
// rounding to bf16 at the end does not depend on the order. Scores are sums of d products of two
// bf16 values, exact products, added in 64 bits too: which of two blocks is chosen then does not
// hang on the order of the additions, and a plain program gets the same lists.
//
// Measured, 6 heads of 86400 tokens of 96, 68 of 675 blocks each: means 16.5 us for 100 MB (6 TB/s), lists
// 40 (reading q takes 20 at the rate of a copy; the rest is the choice, during which memory idles: all
// workgroups are resident at once and in the same phase). One token of 4 sequences, 16 heads on 4 key
// heads, 32 of 256 blocks: 10.5 us, the latency of a chain of means, scores, counts and bounds.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <stdint.h>

#include "block_launch.h"
#include "tile_common.h"

namespace ta {
namespace {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreadsL = 256;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Sum in 64 bits of rows [0, n_rows) of d values, added to acc of this thread's 8 columns: thread t
// takes 16-byte piece t % (d / 8) of rows t / (d / 8), + kRows, ... Two fp64 additions per dword.
template <int D>
struct ColumnSums {
  static constexpr int kPieces = D / 8;
  static constexpr int kRows = kThreadsL / kPieces;
  double acc[8];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.0;
  }
  __device__ __forceinline__ void add(const uint16_t* x, int n_rows) {
    const int piece = threadIdx.x % kPieces, row0 = threadIdx.x / kPieces;
    if (row0 >= kRows) return;
    constexpr int kUnroll = (kBlock + kRows - 1) / kRows;  // a block's rows in one go
    u32x4 w[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int r = row0 + i * kRows;
      w[i] = u32x4{0u, 0u, 0u, 0u};
      if (r < n_rows) w[i] = load16(x + (size_t)r * D + 8 * piece);
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[2 * e] += (double)bf16_lo(w[i][e]);
        acc[2 * e + 1] += (double)bf16_hi(w[i][e]);
      }
  }
  // The totals over all threads' rows: thread c < D returns column c's. part: kRows * D doubles.
  __device__ __forceinline__ double total(double* part) {
    const int piece = threadIdx.x % kPieces, row0 = threadIdx.x / kPieces;
    if (row0 < kRows) {
#pragma unroll
      for (int e = 0; e < 8; ++e) part[row0 * D + 8 * piece + e] = acc[e];
    }
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x < D) {
#pragma unroll
      for (int r = 0; r < kRows; ++r) s += part[r * D + threadIdx.x];
    }
    return s;
  }
};

// The mean of `count` values as the nearest bf16 (0 of none). On the way through fp32 what is not exact
// goes to the neighbour with an odd last bit, which lies on the same side of every tie of bf16 as the
// number itself: a plain conversion to fp32 could land on a tie, and whether the compiler joins the two
// conversions into one hangs on its settings.
__device__ __forceinline__ __bf16 mean_bf16(double sum, int count) {
  if (count <= 0) return (__bf16)0.f;
  const double x = sum / (double)count, ax = fabs(x);
  const float f = (float)x;
  const double af = fabs((double)f);
  uint32_t u = __float_as_uint(f);
  if ((u & 1) == 0 && (af < ax || af > ax)) u += af < ax ? 1u : ~0u;
  return (__bf16)__uint_as_float(u);
}

template <int D>
__global__ __launch_bounds__(kThreadsL) void block_means_kernel(const MeansArgs a) {
  __shared__ double part[ColumnSums<D>::kRows * D];
  const int j = blockIdx.x % a.nb;
  const int bh = blockIdx.x / a.nb, b = bh / a.H;
  const int len = a.lens ? min(max(a.lens[b], 0), a.S) : a.S;
  const int n = min(max(len - j * kBlock, 0), kBlock);
  ColumnSums<D> sums;
  sums.clear();
  sums.add(a.x + ((size_t)bh * a.S + (size_t)j * kBlock) * D, n);
  const double s = sums.total(part);
  if (threadIdx.x < D)
    a.means[((size_t)bh * a.nb + j) * D + threadIdx.x] = __builtin_bit_cast(uint16_t, mean_bf16(s, n));
}

// Orders this wave's LDS accesses (they finish in order; the compiler must not move them).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A score as a number whose order as an unsigned integer is the score's: 0 is kept for blocks that
// may not be chosen, 1 stands for NaN, all ones for forced blocks. -0 and 0 are the same score.
template <typename Key>
constexpr Key kForced = ~(Key)0;

__device__ __forceinline__ uint32_t score_key(float s) {
  if (s != s) return 1;
  const uint32_t u = __float_as_uint(s + 0.f);
  return (u >> 31) ? ~u : (u | (1u << 31));
}
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return 1;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  return (u >> 63) ? ~u : (u | (1ull << 63));
}
// The score behind a 32-bit key (NaN for the keys 0 and 1 that stand for none).
__device__ __forceinline__ float key_score(uint32_t key) {
  if (key <= 1) return __builtin_nanf("");
  return __uint_as_float((key >> 31) ? key ^ (1u << 31) : ~key);
}
__device__ __forceinline__ int leading_zeros(uint32_t x) { return __clz((int)x); }
__device__ __forceinline__ int leading_zeros(uint64_t x) { return __clzll((long long)x); }
template <typename Key>
__device__ __forceinline__ Key lesser(Key a, Key b) { return a < b ? a : b; }
template <typename Key>
__device__ __forceinline__ Key greater(Key a, Key b) { return a > b ? a : b; }

// One workgroup (8 waves) forms the lists of R <= 8 query blocks of one (batch, key head):
//   means    a wave (or more, where the lists are few) per list sums its rows' columns, 64 lanes on
//            16-byte pieces; the means lie in LDS as bf16;
//   scores   on the bf16 matrix cores, 16 rows by 16 key blocks a wave at a time: products are
//            exact, their fp32 sum is off by at most e = d 2^-22 |q|_1 max|k|;
//   choice   a wave per list finds the n_list-th largest score T: a histogram of 256 bins between the
//            smallest and the largest, then of the bin it lies in, until a bin is taken whole. Blocks
//            above T + 2 e are chosen and those below T - 2 e are not, whatever their sums' errors; the
//            few between get their scores in 64 bits, and the best of them are taken. (Where more than
//            64 lie between, as with equal means, all are, in every sweep.)
// (64-bit matrix instructions run at 1/32 of the rate: with them the scores of 4050 lists of 675 blocks
// took 55 us by themselves.)
constexpr int kThreadsM = 512, kWavesM = kThreadsM / 64, kMaxRows = 16;

// The column sums of rows [f0, f1) of all heads' rows (`rows` of each head, head_step apart, head after
// head), one wave: lane l takes piece l % P of rows l / P, + 64 / P, ...; the row groups' sums meet by
// shuffles. Lanes below P end with 8 columns each.
template <int D>
__device__ __forceinline__ void wave_sums(const uint16_t* x, int rows, int64_t f0, int64_t f1, size_t head_step,
                                          int lane, double (&sum)[8]) {
  constexpr int P = D / 8, kGroups = 64 / P, kUnroll = D == 96 ? 13 : 16;  // a block's rows in one or two goes
  const int piece = lane % P, group = lane / P;
  double acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0;
  for (int u = (int)(f0 / rows); u * (int64_t)rows < f1; ++u) {
    const uint16_t* head = x + (size_t)u * head_step * D + 8 * piece;
    const int begin = (int)max(f0 - u * (int64_t)rows, (int64_t)0), end = (int)min(f1 - u * (int64_t)rows, (int64_t)rows);
    for (int r0 = begin; r0 < end; r0 += kGroups * kUnroll) {
      u32x4 w[kUnroll];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        const int r = r0 + i * kGroups + group;
        w[i] = u32x4{0u, 0u, 0u, 0u};
        if (r < end && group < kGroups) w[i] = load16(head + (size_t)r * D);
      }
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        if (r0 + i * kGroups >= end) break;  // additions in 64 bits are slow: none for rows that are not there
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[2 * e] += (double)bf16_lo(w[i][e]);
          acc[2 * e + 1] += (double)bf16_hi(w[i][e]);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sum[e] = acc[e];
#pragma unroll
    for (int k = 1; k < kGroups; ++k) sum[e] += __shfl(acc[e], (lane + k * P) & 63);
  }
}

// <q, k> of two bf16 rows in 64 bits, 64 dims of k read ahead at a time (q lies in LDS).
template <int D>
__device__ __forceinline__ double score64(const uint16_t* k, const uint16_t* q) {
  double s = 0.0;
#pragma unroll 1
  for (int c = 0; c < D; c += 64) {
    u32x4 x[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) x[p] = load16(k + min(c + 8 * p, D - 8));
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      if (D % 64 != 0 && c + 8 * p >= D) break;
      const u32x4 y = load16(q + c + 8 * p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s = __builtin_fma((double)bf16_lo(x[p][e]), (double)bf16_lo(y[e]), s);
        s = __builtin_fma((double)bf16_hi(x[p][e]), (double)bf16_hi(y[e]), s);
      }
    }
  }
  return s;
}

// Inclusive scan over the wave's lanes in ascending order by the vector ALU's lane shifts: within rows
// of 16, then the rows' last lanes handed on. `none` is the operation's identity.
template <typename Op>
__device__ __forceinline__ uint32_t lane_scan(uint32_t x, uint32_t none, Op&& op) {
#define TA_STEP(ctrl, rows) x = op(x, (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, ctrl, rows, 0xf, false))
  TA_STEP(0x111, 0xf);  // row_shr:1
  TA_STEP(0x112, 0xf);
  TA_STEP(0x114, 0xf);
  TA_STEP(0x118, 0xf);
  TA_STEP(0x142, 0xa);  // row_bcast:15
  TA_STEP(0x143, 0xc);  // row_bcast:31
#undef TA_STEP
  return x;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }
__device__ __forceinline__ uint32_t least_of(uint32_t x) {
  return last_lane(lane_scan(x, ~0u, [](uint32_t a, uint32_t b) { return min(a, b); }));
}
__device__ __forceinline__ uint32_t most_of(uint32_t x) {
  return last_lane(lane_scan(x, 0u, [](uint32_t a, uint32_t b) { return max(a, b); }));
}
__device__ __forceinline__ uint64_t least_of(uint64_t x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x = lesser(x, (uint64_t)__shfl_xor((long long)x, s));
  return x;
}
__device__ __forceinline__ uint64_t most_of(uint64_t x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x = greater(x, (uint64_t)__shfl_xor((long long)x, s));
  return x;
}

// A list's keys in LDS, padded with 0 to whole sweeps; fn(j, key) for every key, lane by lane in
// ascending order, four reads ahead of their use.
constexpr int kSweep = 256;
__host__ __device__ __forceinline__ int key_stride(int nb) { return (nb + kSweep - 1) / kSweep * kSweep; }
template <typename Key, typename Fn>
__device__ __forceinline__ void sweep(const Key* kr, int stride, int lane, Fn&& fn) {
  for (int j0 = 0; j0 < stride; j0 += kSweep) {
    Key k[kSweep / 64];
#pragma unroll
    for (int x = 0; x < kSweep / 64; ++x) k[x] = kr[j0 + 64 * x + lane];
#pragma unroll
    for (int x = 0; x < kSweep / 64; ++x) fn(j0 + 64 * x + lane, k[x]);
  }
}

// Blocks below `end` may be chosen; the first `sink` and [near0, near1) of them are.
struct Gate {
  int end, near0, near1;
  __device__ __forceinline__ bool forced(int j, int sink) const { return j < sink || (j >= near0 && j < near1); }
};

// A list's keys in 64 bits, formed anew in every sweep.
template <int D>
struct Keys64 {
  const uint16_t *km, *q;
  Gate gate;
  int sink;
};
template <int D, typename Fn>
__device__ __forceinline__ void sweep(const Keys64<D>& k, int stride, int lane, Fn&& fn) {
  for (int j = lane; j < stride; j += 64) {
    uint64_t key = 0;
    if (j < k.gate.end)
      key = k.gate.forced(j, k.sink) ? kForced<uint64_t> : score_key(score64<D>(k.km + (size_t)j * D, k.q));
    fn(j, key);
  }
}

// One wave: the bar of the n largest of the keys > 0, of which kForced come first: those >= bar are
// chosen, or where ties > 0 those > bar and the first `ties` of those equal to it. False where the
// choice does not depend on scores. hist: 256 words of this wave's.
template <typename Key, typename Keys>
__device__ __forceinline__ bool find_bar(const Keys& kr, int stride, int n, uint32_t* hist, int lane, Key& bar,
                                         int& ties) {
  constexpr Key kTop = kForced<Key>;
  int able = 0, forced = 0;
  Key low = kTop, high = 0;
  sweep(kr, stride, lane, [&](int, Key key) {
    able += __popcll(__builtin_amdgcn_ballot_w64(key != 0));
    forced += __popcll(__builtin_amdgcn_ballot_w64(key == kTop));
    if (key != 0 && key != kTop) {
      low = lesser(low, key);
      high = greater(high, key);
    }
  });
  bar = 1;
  ties = 0;
  if (able <= n) return false;
  int need = n - forced;
  if (need <= 0) {
    bar = kTop;
    ties = need < 0 ? n : 0;
    return false;
  }
  low = least_of(low);
  high = most_of(high);
  Key width = high - low;  // the bar lies in [low, low + width]
  int shift = max(0, (int)(8 * sizeof(Key) - 8) - leading_zeros((Key)(width | 1)));
  for (;;) {
#pragma unroll
    for (int x = 0; x < 4; ++x) hist[lane + 64 * x] = 0;
    wave_sync();
    sweep(kr, stride, lane, [&](int, Key key) {
      if (key >= low && key - low <= width) atomicAdd(&hist[(uint32_t)((key - low) >> shift)], 1u);
    });
    wave_sync();
    // Lane l holds bins 255 - 4 l downwards; above = keys in the bins past its own.
    uint32_t in[4], own = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) own += in[x] = hist[255 - 4 * lane - x];
    uint32_t above = lane_scan(own, 0u, [](uint32_t a, uint32_t b) { return a + b; }) - own;
    int bin = -1, in_bin = 0, left = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (above < (uint32_t)need && above + in[x] >= (uint32_t)need) {
        bin = 255 - 4 * lane - x;
        in_bin = (int)in[x];
        left = need - (int)above;
      }
      above += in[x];
    }
    const int src = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(bin >= 0)) - 1;
    bin = __builtin_amdgcn_readlane(bin, src);
    in_bin = __builtin_amdgcn_readlane(in_bin, src);
    need = __builtin_amdgcn_readlane(left, src);
    bar = low + ((Key)bin << shift);
    if (in_bin == need) return true;  // the whole bin is chosen
    if (shift == 0) {                 // equal keys
      ties = need;
      return true;
    }
    low = bar;
    width = lesser((Key)(((Key)1 << shift) - 1), (Key)(high - low));  // past `high` lie the forced blocks' keys
    shift = max(0, shift - 8);
  }
}

template <int D>
__global__ __launch_bounds__(kThreadsM) void block_lists_kernel(const ListsArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint16_t qm[];         // [16][D]
  uint32_t* hists = reinterpret_cast<uint32_t*>(qm + kMaxRows * D);    // [8][256]; before, 8 maxima
  uint32_t* keys = hists + kWavesM * 256;                              // [R][stride], 0 past nb
  constexpr int kC = D / 32;
  const BlockGeo& g = a.g;
  const int R = a.rows, groups = (g.nq + R - 1) / R, stride = key_stride(g.nb);
  const int i0 = (int)(blockIdx.x % groups) * R;
  const int bh = blockIdx.x / groups, b = bh / g.Hkv, h = bh - b * g.Hkv;
  const int len = g.lens ? min(max(g.lens[b], 0), g.Skv) : g.Skv;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  // Valid rows of query block i.
  auto rows_of = [&](int i) {
    return i < g.nq ? min(max(len - g.off - i * kBlock, 0), min(kBlock, g.Sq - i * kBlock)) : 0;
  };

  // The blocks that query block i may choose, and those it must.
  auto gate_of = [&](int i) {
    const int rows = rows_of(i);
    if (rows == 0) return Gate{0, 0, 0};
    const int first = g.off + i * kBlock, lo = first / kBlock, hi = (first + rows - 1) / kBlock;
    const int end = min((len + kBlock - 1) / kBlock, g.causal ? hi + 1 : g.nb);
    if (a.local == 0) return Gate{end, 0, 0};
    return Gate{end, lo - a.local + 1, g.causal ? hi + 1 : hi + a.local};
  };

  // The key means of a wave's first 16 blocks are on their way while the queries' form.
  const uint16_t* km = a.kmeans + (size_t)bh * g.nb * D;
  u32x4 next[kC];
  auto load = [&](int j) {
#pragma unroll
    for (int c = 0; c < kC; ++c) next[c] = load16(km + (size_t)min(j, g.nb - 1) * D + 32 * c + 8 * (lane >> 4));
  };
  load(16 * wave + (lane & 15));
  {
    // 8 / R waves a list (a power of two), each with a part of the rows of all heads; their sums meet in
    // LDS. (A part of every head's rows left a single token's heads to one wave, one after the other, and
    // its row's sums among zeros took 5 us.)
    double* part = reinterpret_cast<double*>(hists);  // [8][D]
    const int share = R == 1 ? 3 : R == 2 ? 2 : R <= 4 ? 1 : 0;  // log2 of a list's waves
    const int r = wave >> share, p = wave & ((1 << share) - 1), rows = r < R ? rows_of(i0 + r) : 0;
    const int64_t all = (int64_t)rows * g.G, t0 = (all * p) >> share, t1 = (all * (p + 1)) >> share;
    double sum[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
    if (t1 > t0)
      wave_sums<D>(a.q + (((size_t)b * g.H + (size_t)h * g.G) * g.Sq + (size_t)(i0 + r) * kBlock) * D, rows, t0, t1,
                   (size_t)g.Sq, lane, sum);
    if (lane < D / 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) part[wave * D + 8 * lane + e] = sum[e];
    }
    __syncthreads();
    for (int x = tid; x < kMaxRows * D; x += kThreadsM) {
      const int row = x / D, c = x - row * D;
      double total = 0.0;
      if (row < R)
        for (int y = 0; y < 1 << share; ++y) total += part[((row << share) + y) * D + c];
      qm[x] = __builtin_bit_cast(uint16_t, mean_bf16(total, row < R ? rows_of(i0 + row) * g.G : 0));
    }
    __syncthreads();
  }

  {
    const int n = lane & 15, k = lane >> 4;
    bf16x8 qa[kC];
#pragma unroll
    for (int c = 0; c < kC; ++c) qa[c] = as_bf16x8(load16(qm + n * D + 32 * c + 8 * k));
    Gate gates[4];  // of this lane's four rows of the 16
#pragma unroll
    for (int x = 0; x < 4; ++x) gates[x] = gate_of(i0 + 4 * k + x);
    u16x2 mosts = {0, 0};  // the largest magnitudes of key means, even and odd dims apart
    for (int j0 = 16 * wave; j0 < stride; j0 += 16 * kWavesM) {
      const int j = j0 + n;
      u32x4 w[kC];
#pragma unroll
      for (int c = 0; c < kC; ++c) w[c] = next[c];
      load(j + 16 * kWavesM);
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qa[c], as_bf16x8(w[c]), s, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          mosts = __builtin_elementwise_max(mosts, __builtin_bit_cast(u16x2, w[c][e] & 0x7fff7fffu));
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int r = 4 * k + x;
        if (r < R)
          keys[(size_t)r * stride + j] = j >= gates[x].end ? 0u : gates[x].forced(j, a.sink) ? kForced<uint32_t> : score_key(s[x]);
      }
    }
    const uint32_t most = most_of((uint32_t)max(mosts[0], mosts[1]) << 16);  // as the bits of an fp32
    if (lane == 0) hists[wave] = most;
  }
  __syncthreads();
  uint32_t most = 0;
#pragma unroll
  for (int x = 0; x < kWavesM; ++x) most = max(most, hists[x]);
  __syncthreads();

  uint32_t* hist = hists + wave * 256;
  for (int r = wave; r < R; r += kWavesM) {
    const int i = i0 + r;
    if (i >= g.nq) break;
    uint32_t* kr = keys + (size_t)r * stride;
    int32_t* out = a.lists + ((size_t)bh * g.nq + i) * g.n_list;
    int count = 0, tied = 0;
    const uint64_t below = (1ull << lane) - 1;
    // Writes the chosen blocks: keys >= bar, or those > bar and the first `ties` equal to it.
    auto emit = [&](const auto& row, auto bar, int ties) {
      sweep(row, stride, lane, [&](int j, auto key) {
        bool take;
        if (ties > 0) {
          const uint64_t eq = __builtin_amdgcn_ballot_w64(key == bar);
          take = key > bar || (key == bar && tied + __popcll(eq & below) < ties);
          tied += __popcll(eq);
        } else {
          take = key >= bar;
        }
        const uint64_t m = __builtin_amdgcn_ballot_w64(take);
        if (take) out[count + __popcll(m & below)] = j;
        count += __popcll(m);
      });
    };
    uint32_t bar;
    int ties;
    if (find_bar<uint32_t>((const uint32_t*)kr, stride, g.n_list, hist, lane, bar, ties)) {
      // The smallest chosen score, and how far the sums may be off.
      uint32_t least = kForced<uint32_t>;
      sweep(kr, stride, lane, [&](int, uint32_t key) { least = lesser(least, key >= bar ? key : kForced<uint32_t>); });
      float l1 = 0.f;
      for (int x = lane; x < D; x += 64) l1 += fabsf(bf16_lo(qm[r * D + x]));
      least = least_of(least);
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) l1 += __shfl_xor(l1, x);
      // 1.01: the bound's own rounding.
      const float t = key_score(least), off = 1.01f * (2.f * D * 0x1p-22f * l1 * __uint_as_float(most) + 1e-30f);
      const float over = t + off * 1.01f + fabsf(t) * 0x1p-22f, under = t - off * 1.01f - fabsf(t) * 0x1p-22f;
      // Blocks past the bound are settled (all ones: chosen, 0: not); the open ones' indices go to
      // hist. Written so that NaN (of a score, the bar or the bound) leaves a block open.
      int sure = 0, open = 0;
      sweep(kr, stride, lane, [&](int j, uint32_t key) {
        const float v = key_score(key);
        const bool in = key == kForced<uint32_t> || (key != 0 && v > over), out_ = key == 0 || v < under;
        const bool left = !in && !out_;
        const uint64_t m = __builtin_amdgcn_ballot_w64(left);
        const int at = open + __popcll(m & below);
        if (left && at < 64) hist[at] = (uint32_t)j;
        open += __popcll(m);
        sure += __popcll(__builtin_amdgcn_ballot_w64(in));
        kr[j] = in ? kForced<uint32_t> : left ? 1u : 0u;
      });
      wave_sync();
      const int need = g.n_list - sure;
      if (open > 64) {
        // Many blocks too near each other (equal means, infinities): all scores in 64 bits.
        const Keys64<D> all{km, qm + r * D, gate_of(i), a.sink};
        uint64_t bar64;
        find_bar<uint64_t>(all, stride, g.n_list, hist, lane, bar64, ties);
        emit(all, bar64, ties);
      } else {
        if (open > need) {
          // The `need` best of the open blocks by their scores in 64 bits, a lane each; they lie in
          // ascending order, so equal scores go by the lane.
          const int j = lane < open ? (int)hist[lane] : 0;
          uint64_t key = lane < open ? score_key(score64<D>(km + (size_t)j * D, qm + r * D)) : 0;
          int rank = 0;
          for (int x = 0; x < open; ++x) {
            const uint64_t other = (uint64_t)__shfl((long long)key, x);
            rank += other > key || (other == key && x < lane);
          }
          if (lane < open && rank >= need) kr[j] = 0;
          wave_sync();
        }
        emit((const uint32_t*)kr, 1u, 0);
      }
    } else {
      emit((const uint32_t*)kr, bar, ties);
    }
    for (int x = count + lane; x < g.n_list; x += 64) out[x] = -1;
  }
}

template <int D>
size_t lists_lds(int rows, int nb) {
  return (size_t)rows * key_stride(nb) * 4 + kMaxRows * D * 2 + kWavesM * 256 * 4;
}
template <int D>
hipError_t lists_for(const ListsArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)a.g.B * a.g.Hkv * ((a.g.nq + a.rows - 1) / a.rows));
  block_lists_kernel<D><<<grid, kThreadsM, lists_lds<D>(a.rows, a.g.nb), s>>>(a);
  return hipGetLastError();
}

}  // namespace

// The keys of a workgroup's lists lie in LDS, 4 bytes a block: 65 KB of 160 for one list of 16384. Up
// to 8 lists share a workgroup, one a wave (4050 lists of 675 blocks: 5 a workgroup 55 us, 8 40, 16, a
// matrix instruction's rows, 55), fewer where that leaves compute units without one.
static int lists_per_workgroup(int64_t lists, int nb) {
  const int64_t fit = (160 * 1024 - 13 * 1024) / (4 * (int64_t)key_stride(nb));
  return (int)std::max<int64_t>(1, std::min<int64_t>({fit, kWavesM, (lists + 255) / 256}));
}

hipError_t launch_block_means(const MeansArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)((int64_t)a.B * a.H * a.nb);
  if (a.d == 64) block_means_kernel<64><<<grid, kThreadsL, 0, stream>>>(a);
  else if (a.d == 96) block_means_kernel<96><<<grid, kThreadsL, 0, stream>>>(a);
  else block_means_kernel<128><<<grid, kThreadsL, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_block_lists(ListsArgs a, hipStream_t stream) {
  a.rows = std::min(a.g.nq, lists_per_workgroup((int64_t)a.g.B * a.g.Hkv * a.g.nq, a.g.nb));
  if (a.g.d == 64) return lists_for<64>(a, stream);
  if (a.g.d == 96) return lists_for<96>(a, stream);
  return lists_for<128>(a, stream);
}

}  // namespace ta
