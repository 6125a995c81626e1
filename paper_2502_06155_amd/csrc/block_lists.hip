// gfx950 (MI355X, CDNA4) kernels that choose key blocks: block means and lists.
//
// The mean of a block is summed in 64 bits: bf16 values have 8-bit significands, so a sum of up
// to a few thousand of them is exact unless their magnitudes span more than 2^30, and the one
// rounding to bf16 at the end does not depend on the order. Scores are sums of d products of two
// bf16 values, exact products, added in 64 bits too: which of two blocks is chosen then does not
// hang on the order of the additions, and a plain program gets the same lists.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <stdint.h>

#include "block_launch.h"
#include "tile_common.h"

namespace ta {
namespace {

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

// The mean of `count` values as a bf16 (0 of none).
__device__ __forceinline__ __bf16 mean_bf16(double sum, int count) {
  return count > 0 ? (__bf16)(float)(sum / (double)count) : (__bf16)0.f;
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
// may not be chosen, 1 stands for NaN, ~0 for forced blocks. -0 and 0 are the same score.
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return 1;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  return (u >> 63) ? ~u : (u | (1ull << 63));
}

// One workgroup forms the lists of R query blocks of one (batch, key head): the means of their
// rows, the scores (a thread takes key blocks t, t + 256, ...; q's means come from LDS, 64-bit
// FMAs are the work), then a wave per list finds the n_list-th largest key digit by digit with a
// histogram of 256 bins and writes the chosen blocks in ascending order.
template <int D, int R>
__global__ __launch_bounds__(kThreadsL) void block_lists_kernel(const ListsArgs a) {
  extern __shared__ double smem[];
  double* qm = smem;                                            // [R][D]
  double* part = qm + R * D;                                    // column sums, then the histograms
  uint64_t* keys = reinterpret_cast<uint64_t*>(part + ColumnSums<D>::kRows * D);  // [R][nb]
  const BlockGeo& g = a.g;
  const int groups = (g.nq + R - 1) / R;
  const int i0 = (int)(blockIdx.x % groups) * R;
  const int bh = blockIdx.x / groups, b = bh / g.Hkv, h = bh - b * g.Hkv;
  const int len = g.lens ? min(max(g.lens[b], 0), g.Skv) : g.Skv;
  const int tid = threadIdx.x;

#pragma unroll 1
  for (int r = 0; r < R; ++r) {
    const int i = i0 + r;
    const int rows = i < g.nq ? min(max(len - g.off - i * kBlock, 0), min(kBlock, g.Sq - i * kBlock)) : 0;
    ColumnSums<D> sums;
    sums.clear();
    if (rows > 0)
      for (int u = 0; u < g.G; ++u)
        sums.add(a.q + (((size_t)b * g.H + (size_t)h * g.G + u) * g.Sq + (size_t)i * kBlock) * D, rows);
    const double s = sums.total(part);
    if (tid < D) qm[r * D + tid] = (double)(float)mean_bf16(s, rows * g.G);
    __syncthreads();
  }

  const uint16_t* km = a.kmeans + (size_t)bh * g.nb * D;
  for (int j = tid; j < g.nb; j += kThreadsL) {
    double acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = 0.0;
#pragma unroll 2
    for (int p = 0; p < D / 8; ++p) {
      const u32x4 w = load16(km + (size_t)j * D + 8 * p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double lo = (double)bf16_lo(w[e]), hi = (double)bf16_hi(w[e]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          acc[r] = __builtin_fma(lo, qm[r * D + 8 * p + 2 * e], acc[r]);
          acc[r] = __builtin_fma(hi, qm[r * D + 8 * p + 2 * e + 1], acc[r]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = i0 + r;
      const int rows = i < g.nq ? min(max(len - g.off - i * kBlock, 0), min(kBlock, g.Sq - i * kBlock)) : 0;
      uint64_t key = 0;
      if (rows > 0) {
        const int first = g.off + i * kBlock, last = first + rows - 1;
        const int lo = first / kBlock, hi = last / kBlock;
        const bool able = j * kBlock < len && (!g.causal || j <= hi);
        const bool near = a.local > 0 && j > lo - a.local && (g.causal ? j <= hi : j < hi + a.local);
        if (able) key = (j < a.sink || near) ? ~0ull : score_key(acc[r]);
      }
      keys[(size_t)r * g.nb + j] = key;
    }
  }
  __syncthreads();

  const int wave = tid >> 6, lane = tid & 63;
  uint32_t* hist = reinterpret_cast<uint32_t*>(part) + wave * 256;
  for (int r = wave; r < R; r += kThreadsL / 64) {
    const int i = i0 + r;
    if (i >= g.nq) continue;
    const uint64_t* kr = keys + (size_t)r * g.nb;
    int32_t* out = a.lists + ((size_t)bh * g.nq + i) * g.n_list;
    // The keys > 0 are the blocks that may be chosen.
    int able = 0;
    for (int j0 = 0; j0 < g.nb; j0 += 64)
      able += __popcll(__builtin_amdgcn_ballot_w64(j0 + lane < g.nb && kr[j0 + lane] != 0));
    uint64_t bar = 1;   // keys >= bar are chosen ...
    int ties = 0;       // ... or where > 0: keys > bar, and the first `ties` of those equal to it
    if (able > g.n_list) {
      int need = g.n_list;
      uint64_t head = 0;  // the digits found so far
      for (int shift = 56; shift >= 0; shift -= 8) {
#pragma unroll
        for (int x = 0; x < 4; ++x) hist[lane + 64 * x] = 0;
        wave_sync();
        for (int j = lane; j < g.nb; j += 64) {
          const uint64_t key = kr[j];
          if (key != 0 && (shift == 56 || (key >> (shift + 8)) == head))
            atomicAdd(&hist[(uint32_t)(key >> shift) & 255u], 1u);
        }
        wave_sync();
        // Lane l holds bins 4 l .. 4 l + 3; above = keys in the bins past its own.
        uint32_t n[4], own = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) own += n[x] = hist[4 * lane + x];
        uint32_t upto = own;  // bins of lanes >= this one
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
          const uint32_t y = __shfl_down(upto, s);
          if (lane + s < 64) upto += y;
        }
        uint32_t above = upto - own;
        int bin = -1, in_bin = 0, left = 0;
#pragma unroll
        for (int x = 3; x >= 0; --x) {
          if (above < (uint32_t)need && above + n[x] >= (uint32_t)need) {
            bin = 4 * lane + x;
            in_bin = (int)n[x];
            left = need - (int)above;
          }
          above += n[x];
        }
        const int src = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(bin >= 0)) - 1;
        bin = __shfl(bin, src);
        in_bin = __shfl(in_bin, src);
        need = __shfl(left, src);
        head = (head << 8) | (uint64_t)bin;
        if (in_bin == need) {  // the whole bin is chosen: every key of this head on
          bar = head << shift;
          ties = 0;
          break;
        }
        if (shift == 0) {
          bar = head;
          ties = need;
        }
      }
    }
    int count = 0, tied = 0;
    const uint64_t below = (1ull << lane) - 1;
    for (int j0 = 0; j0 < g.nb; j0 += 64) {
      const uint64_t key = j0 + lane < g.nb ? kr[j0 + lane] : 0;
      bool take;
      if (ties > 0) {
        const uint64_t eq = __builtin_amdgcn_ballot_w64(key == bar);
        take = key > bar || (key == bar && tied + __popcll(eq & below) < ties);
        tied += __popcll(eq);
      } else {
        take = key >= bar;
      }
      const uint64_t m = __builtin_amdgcn_ballot_w64(take);
      if (take) out[count + __popcll(m & below)] = j0 + lane;
      count += __popcll(m);
    }
    for (int x = count + lane; x < g.n_list; x += 64) out[x] = -1;
  }
}

template <int D>
hipError_t lists_for(const ListsArgs& a, int per, unsigned grid, size_t lds, hipStream_t s) {
  switch (per) {
    case 8: block_lists_kernel<D, 8><<<grid, kThreadsL, lds, s>>>(a); break;
    case 4: block_lists_kernel<D, 4><<<grid, kThreadsL, lds, s>>>(a); break;
    case 2: block_lists_kernel<D, 2><<<grid, kThreadsL, lds, s>>>(a); break;
    default: block_lists_kernel<D, 1><<<grid, kThreadsL, lds, s>>>(a);
  }
  return hipGetLastError();
}

template <int D>
size_t lists_lds(int per, int nb) {
  return (size_t)(per * D + ColumnSums<D>::kRows * D + per * nb) * sizeof(double);
}

}  // namespace

// The keys of a workgroup's lists lie in LDS, 8 bytes a block: 131 KB for one list of 16384.
int lists_per_workgroup(int nb) { return nb <= 1024 ? 8 : nb <= 2048 ? 4 : nb <= 4096 ? 2 : 1; }

hipError_t launch_block_means(const MeansArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)((int64_t)a.B * a.H * a.nb);
  if (a.d == 64) block_means_kernel<64><<<grid, kThreadsL, 0, stream>>>(a);
  else if (a.d == 96) block_means_kernel<96><<<grid, kThreadsL, 0, stream>>>(a);
  else block_means_kernel<128><<<grid, kThreadsL, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_block_lists(const ListsArgs& a, hipStream_t stream) {
  const int per = std::min(lists_per_workgroup(a.g.nb), a.g.nq >= 8 ? 8 : a.g.nq >= 4 ? 4 : a.g.nq >= 2 ? 2 : 1);
  const unsigned grid = (unsigned)((int64_t)a.g.B * a.g.Hkv * ((a.g.nq + per - 1) / per));
  if (a.g.d == 64) return lists_for<64>(a, per, grid, lists_lds<64>(per, a.g.nb), stream);
  if (a.g.d == 96) return lists_for<96>(a, per, grid, lists_lds<96>(per, a.g.nb), stream);
  return lists_for<128>(a, per, grid, lists_lds<128>(per, a.g.nb), stream);
}

}  // namespace ta
