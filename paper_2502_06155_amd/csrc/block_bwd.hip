// gfx950 (MI355X, CDNA4) kernels for the gradients of attention over selected blocks.
//
// With P = exp(scale <q, k> - lse) over the pairs the forward kept, dP = <dout, v>, delta =
// <dout, out> and dS = P (dP - delta): dq = scale sum dS k, dk = scale sum dS q and
// dv = sum P dout, the last two over the query rows of all G heads of the group.
//
// Passes, on the caller's stream:
//   prep     base-2 lse (+inf for rows without tokens: their P is 0) and -delta per row; clears the
//            columns.
//   columns  the lists turned round: for every key block a bitmap of the query blocks that list it
//            (one atomic OR per entry: the result does not depend on their order).
//   plan     counts a column's query blocks and cuts long ones (a block that every query keeps)
//            into pieces of at most `entries` query blocks.
//   dq       one workgroup per unit of 128 query rows, over its list's key tiles:
//            S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T; a lane owns one query.
//   dk, dv   one workgroup per piece of a key block (128 keys, 4 waves of 32), over the 64-row
//            tiles of its query blocks and heads: S = Q K^T, dP = dO V^T, dV^T += dO^T P,
//            dK^T += Q^T dS; a lane owns one key.
//   sum      adds the pieces of cut units, in order.
// S and dP are formed in both passes: adding dq up from the key side would take fp32 atomics, whose
// order changes results, and more L2 traffic than the matrix cores' time it saves.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "block_launch.h"
#include "block_tiles.h"

namespace ta {
namespace {

// ---------------------------------------------------------------------------------------------
// prep

constexpr int kPrepRowsB = 64;

template <int D>
__global__ __launch_bounds__(kThreadsB) void block_prep_kernel(const BlockBwdArgs a, int64_t n_rows, int64_t n_words) {
  constexpr int kPieces = D / 8, kPer = kPrepRowsB * kPieces / kThreadsB;
  static_assert(kPrepRowsB * kPieces == kThreadsB * kPer, "whole pieces per thread");
  __shared__ float part[kPrepRowsB * kPieces];
  for (int64_t x = (int64_t)blockIdx.x * kThreadsB + threadIdx.x; x < n_words; x += (int64_t)gridDim.x * kThreadsB)
    a.cols[x] = 0;
  const int64_t row0 = (int64_t)blockIdx.x * kPrepRowsB;
  if (row0 >= n_rows) return;
  const int n = (int)min(n_rows - row0, (int64_t)kPrepRowsB);
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int piece = threadIdx.x + kThreadsB * j;
    float acc = 0.f;
    if (piece < n * kPieces) {
      const bf16x8 x = as_bf16x8(load16(a.out + row0 * D + 8 * piece));
      const bf16x8 y = as_bf16x8(load16(a.dout + row0 * D + 8 * piece));
#pragma unroll
      for (int e = 0; e < 8; ++e) acc = __builtin_fmaf((float)x[e], (float)y[e], acc);
    }
    part[piece] = acc;
  }
  __syncthreads();
  if (threadIdx.x < (unsigned)n) {
    float acc = 0.f;
#pragma unroll
    for (int c = 0; c < kPieces; ++c) acc += part[threadIdx.x * kPieces + c];
    const int64_t r = row0 + threadIdx.x;
    const float l = a.lse[r];
    const bool some = l > -INFINITY;
    a.lse2[r] = some ? l * 1.4426950408889634f : INFINITY;
    a.ndelta[r] = some ? -acc : 0.f;
  }
}

// ---------------------------------------------------------------------------------------------
// columns and plan

__device__ __forceinline__ int query_words(const BlockGeo& g) { return (g.nq + 31) / 32; }

__global__ __launch_bounds__(kThreadsB) void block_columns_kernel(const BlockBwdArgs a, int64_t n_entries) {
  const BlockGeo& g = a.g;
  const int words = query_words(g);
  for (int64_t x = (int64_t)blockIdx.x * kThreadsB + threadIdx.x; x < n_entries; x += (int64_t)gridDim.x * kThreadsB) {
    const uint32_t list = (uint32_t)(x / g.n_list);
    const int j = a.lists[x];
    const int i = (int)(list % g.nq);
    const uint32_t bh = list / g.nq;
    const int len = seq_len(g, (int)(bh / g.Hkv));
    const int first = g.off + i * kBlock, last = min(first + min(kBlock, g.Sq - i * kBlock), len) - 1;
    const int end = last < first ? 0 : min(g.nb, (g.causal ? last : len - 1) / kBlock + 1);
    if (j >= 0 && j < end) atomicOr(&a.cols[((size_t)bh * g.nb + j) * words + (i >> 5)], 1u << (i & 31));
  }
}

// plan[4 x] = query blocks of column x, [4 x + 1] = its pieces, [4 x + 2] = its first slot. Slots
// are handed out by a counter: which ones a column gets may differ from call to call, what it sums
// up and in which order does not.
__global__ __launch_bounds__(kThreadsB) void block_plan_kernel(const BlockBwdArgs a, int64_t n_cols) {
  const int words = query_words(a.g);
  const int64_t x = (int64_t)blockIdx.x * kThreadsB + threadIdx.x;
  if (x >= n_cols) return;
  int n = 0;
  for (int w = 0; w < words; ++w) n += __builtin_popcount(a.cols[x * words + w]);
  const int pieces = max(1, (n + a.entries - 1) / a.entries);
  a.plan[4 * x] = n;
  a.plan[4 * x + 1] = pieces;
  if (pieces > 1) a.plan[4 * x + 2] = atomicAdd(reinterpret_cast<int*>(a.cols + n_cols * words), pieces);
}

// P = exp2(c s - lse2) clamped to [0, 1] (the exponent is <= 0 up to rounding for kept pairs; the
// clamp keeps rows of zeros past a tile's valid range finite, which then add exactly nothing).
__device__ __forceinline__ float prob(float s, float c, float lse2) {
  return __builtin_amdgcn_fmed3f(fast_exp2(__builtin_fmaf(s, c, -lse2)), 0.f, 1.f);
}

// ---------------------------------------------------------------------------------------------
// dq

// dS^T of a 32-key block as the B operand of dQ^T += K^T dS^T; dp holds dP - delta.
__device__ __forceinline__ void score_grads(const f32x16& s, const f32x16& dp, float c, float lse2, bf16x8 (&ds)[2]) {
#pragma unroll
  for (int c2 = 0; c2 < 2; ++c2) {
    f32x8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = prob(s[8 * c2 + e], c, lse2) * dp[8 * c2 + e];
    ds[c2] = __builtin_convertvector(x, bf16x8);
  }
}

template <int D>
__global__ __launch_bounds__(kThreadsB, 2) void block_dq_kernel(const BlockBwdArgs a) {
  using Sh = BlockShape<D>;
  __shared__ uint16_t sK[2][Sh::kTileElems], sV[2][Sh::kTileElems];
  __shared__ uint32_t bits[kBlockWords];
  const BlockGeo& g = a.g;
  const uint32_t lists = (uint32_t)g.B * g.Hkv * g.nq;
  const uint32_t work = xcd_unit(blockIdx.x, lists * a.units * a.pieces_q);
  if (work >= lists * a.units * a.pieces_q) return;
  const int piece = (int)(work % a.pieces_q);
  const uint32_t lu = work / a.pieces_q, list = lu / a.units;
  const int unit = (int)(lu % a.units);
  const int i = (int)(list % g.nq);
  const int bh = (int)(list / g.nq), b = bh / g.Hkv, h = bh - b * g.Hkv;
  const ListRows rows(g, b, h, i);
  const int n_rows = g.G * rows.tokens;
  if (unit * kUnitRows >= n_rows) return;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 31, hf = lane >> 5;
  const int words = (g.nb + 31) / 32;
  list_bits(g, a.lists + (size_t)list * g.n_list, rows, bits, words);

  const int r = unit * kUnitRows + wave * 32 + n;
  int pos = 0;
  const size_t row = rows.global(min(r, n_rows - 1), pos);
  const bool valid = r < n_rows && pos < rows.len;
  const int last = valid ? (g.causal ? pos : rows.len - 1) : -1;
  bf16x8 qf[Sh::kChunks], gf[Sh::kChunks];
  lane_row<D>(a.q + row * D, valid, a.keep, a.flip, hf, qf);
  lane_row<D>(a.dout + row * D, valid, ~0u, 0u, hf, gf);
  const float lse2 = valid ? a.lse2[row] : INFINITY;
  const float ndelta = valid ? a.ndelta[row] : 0.f;
  f32x16 dp_start;
#pragma unroll
  for (int e = 0; e < 16; ++e) dp_start[e] = ndelta;
  f32x16 acc[Sh::kDBlocks];
#pragma unroll
  for (int mb = 0; mb < Sh::kDBlocks; ++mb) acc[mb] = f32x16{};

  KeyTiles nxt;
  nxt.half = 0;
  nxt.end = g.causal ? min(rows.len, rows.last() + 1) : rows.len;
  if (a.pieces_q == 1) {
    nxt.walk.start(bits, words, 0, g.nb);
  } else {
    const int all = count_bits(bits, words);
    const int e0 = (int)((int64_t)all * piece / a.pieces_q), e1 = (int)((int64_t)all * (piece + 1) / a.pieces_q);
    nxt.walk.start(bits, words, e0, e1 - e0);
  }
  if (!nxt.done()) {
    const uint16_t* Kh = a.k + (size_t)bh * g.Skv * D;
    const uint16_t* Vh = a.v + (size_t)bh * g.Skv * D;
    TileLoads<D> ld;
    ld.init(wave, lane);
    RowsAt<D> ra;
    ra.init(n, hf);
    ColsAt<D> ca;
    ca.init(lane);
    int key0 = nxt.key0();
    ld.load(Kh + (size_t)key0 * D, rows.len - key0, sK[0], wave);
    ld.load(Vh + (size_t)key0 * D, rows.len - key0, sV[0], wave);
    nxt.next();
    wait_tile_loads();
    __syncthreads();

    auto both = [&](const uint16_t* tk, const uint16_t* tv, int kb, f32x16& s, f32x16& dp) {
      s = f32x16{};
      dp = dp_start;
#pragma unroll
      for (int cc = 0; cc < Sh::kChunks; ++cc) {
        s = mfma32(rows_frag<D>(tk, ra, kb, cc), qf[cc], s);
        dp = mfma32(rows_frag<D>(tv, ra, kb, cc), gf[cc], dp);
      }
    };
    auto accumulate = [&](const uint16_t* tk, int kb, const bf16x8(&ds)[2]) {
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
        for (int mb = 0; mb < Sh::kDBlocks; ++mb)
          acc[mb] = mfma32(cols_frag<D>(tk, ca, mb, 2 * kb + c2), ds[c2], acc[mb]);
    };
    auto tile_step = [&](auto bufc, bool more) {
      constexpr int buf = decltype(bufc)::value;
      if (more) {
        ld.load(Kh + (size_t)nxt.key0() * D, rows.len - nxt.key0(), sK[buf ^ 1], wave);
        ld.load(Vh + (size_t)nxt.key0() * D, rows.len - nxt.key0(), sV[buf ^ 1], wave);
      }
      const int lim = last - key0;
      if (__builtin_amdgcn_ballot_w64(lim >= 0) != 0) {
        // Block 1's products run while block 0's dS forms, then block 0's update while block 1's
        // dS forms; the fences keep each phase's fragments from moving into the one before.
        const bool mask = __builtin_amdgcn_ballot_w64(lim < kBlockK - 1) != 0;
        f32x16 s0, dp0, s1, dp1;
        bf16x8 ds0[2], ds1[2];
        both(sK[buf], sV[buf], 0, s0, dp0);
        if (mask) mask_keys(s0, 0, hf, lim);
        __builtin_amdgcn_sched_barrier(0);
        both(sK[buf], sV[buf], 1, s1, dp1);
        score_grads(s0, dp0, a.c, lse2, ds0);
        __builtin_amdgcn_sched_barrier(0);
        if (mask) mask_keys(s1, 1, hf, lim);
        accumulate(sK[buf], 0, ds0);
        score_grads(s1, dp1, a.c, lse2, ds1);
        __builtin_amdgcn_sched_barrier(0);
        accumulate(sK[buf], 1, ds1);
      }
      if (more) {
        key0 = nxt.key0();
        nxt.next();
      }
      wait_tile_loads();
      __syncthreads();
    };
    for (;;) {
      bool more = !nxt.done();
      tile_step(std::integral_constant<int, 0>{}, more);
      if (!more) break;
      more = !nxt.done();
      tile_step(std::integral_constant<int, 1>{}, more);
      if (!more) break;
    }
  }

  if (r < n_rows) {
    if (a.pieces_q == 1) {
      store_bf16<D>(a.dq + row * D, acc, a.scale, hf);
    } else {
      store_f32<D>(a.part_q + (((size_t)lu * a.pieces_q + piece) * kUnitRows + wave * 32 + n) * D, acc, a.scale, hf);
    }
  }
}

// Adds the pieces of dq units, in order; a thread takes 4 consecutive d of a row.
template <int D>
__global__ __launch_bounds__(kThreadsB) void block_dq_sum_kernel(const BlockBwdArgs a) {
  const BlockGeo& g = a.g;
  const uint32_t lu = blockIdx.x, list = lu / a.units;
  const int unit = (int)(lu % a.units), i = (int)(list % g.nq);
  const int bh = (int)(list / g.nq), b = bh / g.Hkv, h = bh - b * g.Hkv;
  const ListRows rows(g, b, h, i);
  const int n_rows = g.G * rows.tokens;
  const float* part = a.part_q + (size_t)lu * a.pieces_q * kUnitRows * D;
  for (int x = threadIdx.x; x < kUnitRows * (D / 4); x += kThreadsB) {
    const int rr = x / (D / 4), d0 = 4 * (x % (D / 4)), r = unit * kUnitRows + rr;
    if (r >= n_rows) return;
    int pos;
    const size_t row = rows.global(r, pos);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < a.pieces_q; ++p)
      y += *reinterpret_cast<const f32x4*>(part + ((size_t)p * kUnitRows + rr) * D + d0);
    *reinterpret_cast<u32x2*>(a.dq + row * D + d0) = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
  }
}

// ---------------------------------------------------------------------------------------------
// dk, dv

// The 64-row tiles of a column's query blocks: head after head, half after half.
struct QueryTiles {
  BitWalk walk;
  int head, half, G, off, Sq, len;
  __device__ __forceinline__ bool done() const { return walk.at < 0; }
  __device__ __forceinline__ int first() const { return off + walk.at * kBlock + half * kBlockK; }  // position
  // Valid rows from the tile's first on (rows past the tile's 64 among them).
  __device__ __forceinline__ int valid() const {
    const int i0 = walk.at * kBlock;
    return min(min(kBlock, Sq - i0), len - off - i0) - half * kBlockK;
  }
  __device__ __forceinline__ size_t row0(size_t group_row) const {
    return group_row + (size_t)head * Sq + walk.at * kBlock + half * kBlockK;
  }
  __device__ __forceinline__ void next() {
    if (half == 0 && valid() > kBlockK) {
      half = 1;
      return;
    }
    half = 0;
    if (++head == G) {
      head = 0;
      walk.next();
    }
  }
};

template <int D>
constexpr int dkdv_wgs() { return D == 128 ? 1 : 2; }

template <int D, bool CAUSAL>
__global__ __launch_bounds__(kThreadsB, dkdv_wgs<D>()) void block_dkdv_kernel(const BlockBwdArgs a) {
  using Sh = BlockShape<D>;
  __shared__ uint16_t sQ[2][Sh::kTileElems], sG[2][Sh::kTileElems];
  __shared__ float sL[2][kBlockK], sD[2][kBlockK];
  __shared__ uint32_t bits[kBlockWords];
  const BlockGeo& g = a.g;
  const uint32_t cols = (uint32_t)g.B * g.Hkv * g.nb;
  const uint32_t work = xcd_unit(blockIdx.x, cols * a.pieces_k);
  if (work >= cols * a.pieces_k) return;
  const int piece = (int)(work % a.pieces_k);
  const uint32_t col = work / a.pieces_k;
  const int pieces = a.plan[4 * (size_t)col + 1];
  if (piece >= pieces) return;
  const int all = a.plan[4 * (size_t)col];
  const int j = (int)(col % g.nb);
  const int bh = (int)(col / g.nb), b = bh / g.Hkv, h = bh - b * g.Hkv;
  const int len = seq_len(g, b);
  const size_t group_row = ((size_t)b * g.H + (size_t)h * g.G) * g.Sq;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 31, hf = lane >> 5;
  const int words = query_words(g);
  for (int x = tid; x < words; x += kThreadsB) bits[x] = a.cols[(size_t)col * words + x];
  __syncthreads();

  // This lane's key as the B operand of S = Q K^T and dP = dO V^T.
  const int key = j * kBlock + wave * 32 + n;
  const bool valid = key < len;
  const bool wave_active = j * kBlock + wave * 32 < len;
  const size_t kr = (size_t)bh * g.Skv + key;
  bf16x8 kf[Sh::kChunks], vf[Sh::kChunks];
  lane_row<D>(a.k + kr * D, valid, a.keep, a.flip, hf, kf);
  lane_row<D>(a.v + kr * D, valid, ~0u, 0u, hf, vf);
  f32x16 dk[Sh::kDBlocks], dv[Sh::kDBlocks];
#pragma unroll
  for (int mb = 0; mb < Sh::kDBlocks; ++mb) {
    dk[mb] = f32x16{};
    dv[mb] = f32x16{};
  }

  QueryTiles nxt;
  nxt.head = 0;
  nxt.half = 0;
  nxt.G = g.G;
  nxt.off = g.off;
  nxt.Sq = g.Sq;
  nxt.len = len;
  const int e0 = (int)((int64_t)all * piece / pieces), e1 = (int)((int64_t)all * (piece + 1) / pieces);
  nxt.walk.start(bits, words, e0, e1 - e0);
  if (!nxt.done()) {
    TileLoads<D> ld;
    ld.init(wave, lane);
    RowsAt<D> ra;
    ra.init(n, hf);
    ColsAt<D> ca;
    ca.init(lane);
    // Q, dO, lse2 and -delta of a tile; rows past the valid ones read as zeros and add nothing.
    auto load_tile = [&](const QueryTiles& t, int bi) {
      const size_t row0 = t.row0(group_row);
      const int nv = t.valid();
      ld.load(a.q + row0 * D, nv, sQ[bi], wave);
      ld.load(a.dout + row0 * D, nv, sG[bi], wave);
      if (wave == 0) {
        load_dword_to_lds(buffer_words(a.lse2 + row0, (uint32_t)(nv * 4)), lds_addr((const uint16_t*)sL[bi]), 4 * lane);
        load_dword_to_lds(buffer_words(a.ndelta + row0, (uint32_t)(nv * 4)), lds_addr((const uint16_t*)sD[bi]),
                          4 * lane);
      }
    };
    load_tile(nxt, 0);
    int first = nxt.first();
    nxt.next();
    wait_tile_loads();
    __syncthreads();

    // One tile as a stream of MFMAs, each in a fenced packet with its share of the vector work and
    // its operand read from LDS two packets ahead: S and dP of half 0, S and dP of half 1 with half
    // 0's P and dS forming, the updates of half 0 with half 1's, the updates of half 1. MASK: rows
    // before this lane's key (lim of the tile's rows) get P = 0.
    auto stream = [&](auto bufc, auto maskc, int lim) {
      constexpr int buf = decltype(bufc)::value;
      constexpr bool kMask = decltype(maskc)::value;
      constexpr int kC = Sh::kChunks, kMb = Sh::kDBlocks, kAhead = 2;
      constexpr int kHalf = 2 * kC, kAcc = 4 * kMb, kN = 2 * kHalf + 2 * kAcc, kPerC2 = kAcc / 2;
      f32x16 sc[2], dp[2];
      bf16x8 pb[2][2], db[2][2];
      f32x4 l4[2][4];
      float t0, t1, y0, y1;
      const int low = lim - 4 * hf;
      auto dp_start = [&](int qc, f32x16& x) {
#pragma unroll
        for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const f32x4 d4 = *reinterpret_cast<const f32x4*>(&sD[buf][32 * qc + 16 * c2 + 8 * u + 4 * hf]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[8 * c2 + 4 * u + e] = d4[e];
          }
      };
      auto frag = [&](auto ic) -> bf16x8 {
        constexpr int x = decltype(ic)::value;
        if constexpr (x < 2 * kHalf) {
          constexpr int hh = x / kHalf, y = x % kHalf;
          if constexpr (y < kC) return rows_frag<D>(sQ[buf], ra, hh, y);
          else return rows_frag<D>(sG[buf], ra, hh, y - kC);
        } else {
          constexpr int y = x - 2 * kHalf, hh = y / kAcc, z = y % kAcc, c2 = z / kPerC2, q = z % kPerC2;
          return cols_frag<D>(q % 2 ? sQ[buf] : sG[buf], ca, q / 2, 2 * hh + c2);
        }
      };
      auto mfma = [&](auto ic, const bf16x8& f) {
        constexpr int x = decltype(ic)::value;
        if constexpr (x < 2 * kHalf) {
          constexpr int hh = x / kHalf, y = x % kHalf;
          if constexpr (y < kC) sc[hh] = mfma32(f, kf[y], y == 0 ? f32x16{} : sc[hh]);
          else dp[hh] = mfma32(f, vf[y - kC], dp[hh]);
        } else {
          constexpr int y = x - 2 * kHalf, hh = y / kAcc, z = y % kAcc, c2 = z / kPerC2, q = z % kPerC2, mb = q / 2;
          if constexpr (q % 2) dk[mb] = mfma32(f, db[hh][c2], dk[mb]);
          else dv[mb] = mfma32(f, pb[hh][c2], dv[mb]);
        }
      };
      auto side = [&](auto ic) {
        constexpr int x = decltype(ic)::value;
        if constexpr (x == 0 || x == kHalf) dp_start(x / kHalf, dp[x / kHalf]);
        static_for<8>([&](auto qc) {
          constexpr int hh = decltype(qc)::value / 4, q4 = decltype(qc)::value % 4;
          constexpr int st = hh == 0 ? kHalf : 2 * kHalf, pk = hh == 0 ? kHalf : kAcc;
          constexpr int at = st + ((2 * q4 + 1) * pk + 7) / 8 - 1 - kAhead;
          if constexpr (at == x)
            l4[hh][q4] = *reinterpret_cast<const f32x4*>(&sL[buf][32 * hh + 16 * (q4 / 2) + 8 * (q4 % 2) + 4 * hf]);
        });
        constexpr int hh = x < kHalf ? -1 : (x < 2 * kHalf ? 0 : (x < 2 * kHalf + kAcc ? 1 : -1));
        if constexpr (hh >= 0) {
          constexpr int k = hh == 0 ? x - kHalf : x - 2 * kHalf, kPk = hh == 0 ? kHalf : kAcc;
#pragma unroll
          for (int m = k * 80 / kPk; m < (k + 1) * 80 / kPk; ++m) {
            // Step m % 10 of pair m / 10: entries e, e + 1 are tile rows 32 hh + 16 c2 + 8 u + 4 hf + j.
            const int op = m % 10, e = 2 * (m / 10), c2 = e / 8, u = (e % 8) / 4, jj = e % 4;
            const int rr = 32 * hh + 16 * c2 + 8 * u + jj;
            if (op == 0) {
              t0 = __builtin_fmaf(sc[hh][e], a.c, -l4[hh][2 * c2 + u][jj]);
              if (kMask && rr < low) t0 = -INFINITY;
            }
            if (op == 1) {
              t1 = __builtin_fmaf(sc[hh][e + 1], a.c, -l4[hh][2 * c2 + u][jj + 1]);
              if (kMask && rr + 1 < low) t1 = -INFINITY;
            }
            if (op == 2) t0 = __builtin_amdgcn_fmed3f(fast_exp2(t0), 0.f, 1.f);
            if (op == 4) t1 = __builtin_amdgcn_fmed3f(fast_exp2(t1), 0.f, 1.f);
            if (op == 6) y0 = t0 * dp[hh][e];
            if (op == 7) y1 = t1 * dp[hh][e + 1];
            if (op == 8) {
              u32x4 w = __builtin_bit_cast(u32x4, pb[hh][c2]);
              w[(e % 8) / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{t0, t1}, bf16x2));
              pb[hh][c2] = __builtin_bit_cast(bf16x8, w);
            }
            if (op == 9) {
              u32x4 w = __builtin_bit_cast(u32x4, db[hh][c2]);
              w[(e % 8) / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{y0, y1}, bf16x2));
              db[hh][c2] = __builtin_bit_cast(bf16x8, w);
            }
          }
        }
      };
      bf16x8 fr[kAhead + 1];
      static_for<kAhead>([&](auto jc) { fr[decltype(jc)::value] = frag(jc); });
      __builtin_amdgcn_sched_barrier(0);
      static_for<kN>([&](auto ic) {
        constexpr int x = decltype(ic)::value;
        if constexpr (x + kAhead < kN)
          fr[(x + kAhead) % (kAhead + 1)] = frag(std::integral_constant<int, x + kAhead>{});
        mfma(ic, fr[x % (kAhead + 1)]);
        side(ic);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    auto tile_step = [&](auto bufc, bool more) {
      if (more) load_tile(nxt, decltype(bufc)::value ^ 1);
      if (wave_active) {
        const int lim = CAUSAL ? key - first : 0;  // the tile's first row that attends to this key
        if (CAUSAL && __builtin_amdgcn_ballot_w64(lim > 0) != 0) stream(bufc, std::true_type{}, lim);
        else stream(bufc, std::false_type{}, 0);
      }
      if (more) {
        first = nxt.first();
        nxt.next();
      }
      wait_tile_loads();
      __syncthreads();
    };
    for (;;) {
      bool more = !nxt.done();
      tile_step(std::integral_constant<int, 0>{}, more);
      if (!more) break;
      more = !nxt.done();
      tile_step(std::integral_constant<int, 1>{}, more);
      if (!more) break;
    }
  }

  if (!valid) {  // padding: its K and V rows were zeros, what formed for them counts for nobody
#pragma unroll
    for (int mb = 0; mb < Sh::kDBlocks; ++mb) {
      dk[mb] = f32x16{};
      dv[mb] = f32x16{};
    }
  }
  if (pieces == 1) {
    if (key < g.Skv) {
      store_bf16<D>(a.dk + kr * D, dk, a.scale, hf);
      store_bf16<D>(a.dv + kr * D, dv, 1.f, hf);
    }
  } else {
    const int slot = a.plan[4 * (size_t)col + 2] + piece;
    if (slot < a.slots) {
      float* part = a.part_k + ((size_t)slot * 2 * kBlock + wave * 32 + n) * D;
      store_f32<D>(part, dk, a.scale, hf);
      store_f32<D>(part + (size_t)kBlock * D, dv, 1.f, hf);
    }
  }
}

// Adds the pieces of cut key blocks, in order; dk by blockIdx.y = 0, dv by 1.
template <int D>
__global__ __launch_bounds__(kThreadsB) void block_dkdv_sum_kernel(const BlockBwdArgs a) {
  const BlockGeo& g = a.g;
  const uint32_t col = blockIdx.x;
  const int pieces = a.plan[4 * (size_t)col + 1];
  if (pieces == 1) return;
  const int slot = a.plan[4 * (size_t)col + 2];
  if (slot + pieces > a.slots) return;
  const int j = (int)(col % g.nb);
  const size_t row0 = (size_t)(col / g.nb) * g.Skv + (size_t)j * kBlock;
  const int n_rows = min(kBlock, g.Skv - j * kBlock);
  const float* part = a.part_k + ((size_t)slot * 2 + blockIdx.y) * kBlock * D;
  uint16_t* out = blockIdx.y ? a.dv : a.dk;
  for (int x = threadIdx.x; x < n_rows * (D / 4); x += kThreadsB) {
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < pieces; ++p) y += *reinterpret_cast<const f32x4*>(part + (size_t)p * 2 * kBlock * D + 4 * x);
    *reinterpret_cast<u32x2*>(out + row0 * D + 4 * x) = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
  }
}

template <int D>
hipError_t block_bwd_for(const BlockBwdArgs& a, hipStream_t s) {
  const BlockGeo& g = a.g;
  const int64_t rows = (int64_t)g.B * g.H * g.Sq, cols = (int64_t)g.B * g.Hkv * g.nb;
  const int64_t words = cols * ((g.nq + 31) / 32) + 1;  // the slot counter behind them
  const int64_t lists = (int64_t)g.B * g.Hkv * g.nq, entries = lists * g.n_list;
  block_prep_kernel<D><<<(unsigned)((rows + kPrepRowsB - 1) / kPrepRowsB), kThreadsB, 0, s>>>(a, rows, words);
  block_columns_kernel<<<(unsigned)std::min<int64_t>((entries + kThreadsB - 1) / kThreadsB, 4096), kThreadsB, 0, s>>>(
      a, entries);
  block_plan_kernel<<<(unsigned)((cols + kThreadsB - 1) / kThreadsB), kThreadsB, 0, s>>>(a, cols);
  block_dq_kernel<D><<<xcd_grid((uint32_t)(lists * a.units * a.pieces_q)), kThreadsB, 0, s>>>(a);
  if (a.pieces_q > 1) block_dq_sum_kernel<D><<<(unsigned)(lists * a.units), kThreadsB, 0, s>>>(a);
  const unsigned grid_k = xcd_grid((uint32_t)(cols * a.pieces_k));
  if (g.causal) block_dkdv_kernel<D, true><<<grid_k, kThreadsB, 0, s>>>(a);
  else block_dkdv_kernel<D, false><<<grid_k, kThreadsB, 0, s>>>(a);
  if (a.pieces_k > 1) block_dkdv_sum_kernel<D><<<dim3((unsigned)cols, 2), kThreadsB, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_bwd(const BlockBwdArgs& a, hipStream_t stream) {
  if (a.g.d == 64) return block_bwd_for<64>(a, stream);
  if (a.g.d == 96) return block_bwd_for<96>(a, stream);
  return block_bwd_for<128>(a, stream);
}

}  // namespace ta
