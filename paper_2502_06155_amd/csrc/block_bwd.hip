// gfx950 (MI355X, CDNA4) kernels for the gradients of attention over selected blocks.
//
// With P = exp(scale <q, k> - lse) over the pairs the forward kept, dP = <dout, v>, delta =
// <dout, out> and dS = P (dP - delta): dq = scale sum dS k, dk = scale sum dS q and
// dv = sum P dout, the last two over the query rows of all G heads of the group.
//
// Passes, on the caller's stream:
//   prep     base-2 lse (+inf for rows without tokens: their P is 0) and -delta per row; in the same
//            launch the lists turned round: for every key block a bitmap (its column) of the query
//            blocks that list it, 32 of them a workgroup.
//   plan     counts a column's query blocks, cuts long ones (a block that every query keeps) into
//            pieces of at most `entries` query blocks, and orders the pieces longest first.
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

__device__ __forceinline__ int query_words(const BlockGeo& g) { return (g.nq + 31) / 32; }

// One word of every column of a (batch, key head): the lists of 32 query blocks. Entries that name
// no block, or one that no row of the query block may attend to, are left out as in the forward.
__device__ __forceinline__ void column_words(const BlockBwdArgs& a, uint32_t work, uint32_t* col) {
  const BlockGeo& g = a.g;
  const int words = query_words(g);
  const int w = (int)(work % words);
  const uint32_t bh = work / words;
  const int len = seq_len(g, (int)(bh / g.Hkv));
  for (int j = threadIdx.x; j < g.nb; j += kThreadsB) col[j] = 0;
  __syncthreads();
  const int i0 = 32 * w, n = min(32, g.nq - i0) * g.n_list;
  const int32_t* lists = a.lists + ((size_t)bh * g.nq + i0) * g.n_list;
  for (int x = threadIdx.x; x < n; x += kThreadsB) {
    const int bit = x / g.n_list, i = i0 + bit, j = lists[x];
    const int first = g.off + i * kBlock, last = min(first + min(kBlock, g.Sq - i * kBlock), len) - 1;
    const int end = last < first ? 0 : min(g.nb, (g.causal ? last : len - 1) / kBlock + 1);
    if (j >= 0 && j < end) atomicOr(&col[j], 1u << bit);
  }
  __syncthreads();
  for (int j = threadIdx.x; j < g.nb; j += kThreadsB) a.cols[((size_t)bh * g.nb + j) * words + w] = col[j];
}

template <int D>
__global__ __launch_bounds__(kThreadsB) void block_prep_kernel(const BlockBwdArgs a, int64_t n_rows, uint32_t prep_wgs) {
  constexpr int kPieces = D / 8, kPer = kPrepRowsB * kPieces / kThreadsB;
  static_assert(kPrepRowsB * kPieces == kThreadsB * kPer, "whole pieces per thread");
  extern __shared__ float part[];  // the rows' pieces, or the columns' words
  if (blockIdx.x >= prep_wgs) {
    column_words(a, blockIdx.x - prep_wgs, reinterpret_cast<uint32_t*>(part));
    return;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.counts[8] = 0;
  const int64_t row0 = (int64_t)blockIdx.x * kPrepRowsB;
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
// plan

// One workgroup per XCD cuts the columns of its share into pieces and lists the pieces longest first
// (by 64 sizes): popular blocks' pieces start the launch, and those of blocks that hardly anybody
// lists even out its end. plan[4 col] = the column's query blocks, + 1 = its pieces, + 2 = its first
// slot; items[xcd * cap + i] = {column, piece}; counts[xcd] = items of the share. Slots come from a
// counter and items of one size in any order: where a piece's sums lie and when it runs may differ
// from call to call, what it adds up and in which order does not.
constexpr int kPlanThreads = 1024, kSizes = 64;

__global__ __launch_bounds__(kPlanThreads) void block_plan_kernel(const BlockBwdArgs a, uint32_t cols, uint32_t per) {
  __shared__ int hist[kSizes];
  const int words = query_words(a.g);
  const uint32_t x0 = blockIdx.x * per, x1 = min(cols, x0 + per);
  const int tid = threadIdx.x;
  if (tid < kSizes) hist[tid] = 0;
  __syncthreads();
  // Entries of pieces of one column differ by at most one: one size stands for all.
  auto size_of = [&](int n, int pieces) {
    return kSizes - 1 - min(kSizes - 1, (int)((int64_t)((n + pieces - 1) / pieces) * kSizes / (a.entries + 1)));
  };
  for (uint32_t x = x0 + tid; x < x1; x += kPlanThreads) {
    int n = 0;
    for (int w = 0; w < words; ++w) n += __builtin_popcount(a.cols[(size_t)x * words + w]);
    const int pieces = max(1, (n + a.entries - 1) / a.entries);
    a.plan[4 * (size_t)x] = n;
    a.plan[4 * (size_t)x + 1] = pieces;
    a.plan[4 * (size_t)x + 2] = pieces > 1 ? atomicAdd(&a.counts[8], pieces) : 0;
    atomicAdd(&hist[size_of(n, pieces)], pieces);
  }
  __syncthreads();
  if (tid < kSizes) {  // one wave: where each size starts
    const int own = hist[tid];
    int upto = own;
#pragma unroll
    for (int s = 1; s < kSizes; s <<= 1) {
      const int y = __shfl_up(upto, s);
      if (tid >= s) upto += y;
    }
    hist[tid] = upto - own;
    if (tid == kSizes - 1) a.counts[blockIdx.x] = upto;
  }
  __syncthreads();
  int2* items = reinterpret_cast<int2*>(a.items) + (size_t)blockIdx.x * per * a.pieces_k;
  for (uint32_t x = x0 + tid; x < x1; x += kPlanThreads) {
    const int n = a.plan[4 * (size_t)x], pieces = a.plan[4 * (size_t)x + 1];
    const int at = atomicAdd(&hist[size_of(n, pieces)], pieces);
    for (int p = 0; p < pieces; ++p) items[at + p] = int2{(int)x, p};
  }
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

// The query-side pass of one unit; `id` as a workgroup id.
template <int D>
__device__ __forceinline__ void dq_unit(const BlockBwdArgs& a, uint32_t id, uint16_t (&sK)[2][BlockShape<D>::kTileElems],
                                        uint16_t (&sV)[2][BlockShape<D>::kTileElems], uint32_t (&bits)[kBlockWords]) {
  using Sh = BlockShape<D>;
  const BlockGeo& g = a.g;
  const uint32_t lists = (uint32_t)g.B * g.Hkv * g.nq;
  const uint32_t work = xcd_unit(id, lists * a.units * a.pieces_q);
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

// The key-side pass of one piece of a key block; `id` as a workgroup id: every XCD runs the items of
// its share in the plan's order.
template <int D, bool CAUSAL>
__device__ __forceinline__ void dkdv_unit(const BlockBwdArgs& a, uint32_t id, uint16_t (&sQ)[2][BlockShape<D>::kTileElems],
                                          uint16_t (&sG)[2][BlockShape<D>::kTileElems], float (&sL)[2][kBlockK],
                                          float (&sD)[2][kBlockK], uint32_t (&bits)[kBlockWords]) {
  using Sh = BlockShape<D>;
  const BlockGeo& g = a.g;
  const uint32_t cap = ((uint32_t)g.B * g.Hkv * g.nb + 7) / 8 * (uint32_t)a.pieces_k;
  if (id / 8 >= (uint32_t)a.counts[id % 8]) return;
  const int2 item = reinterpret_cast<const int2*>(a.items)[(size_t)(id % 8) * cap + id / 8];
  const uint32_t col = (uint32_t)item.x;
  const int piece = item.y, pieces = a.plan[4 * (size_t)col + 1];
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
    [[maybe_unused]] int first = nxt.first(), block = nxt.walk.at;
    nxt.next();
    wait_tile_loads();
    __syncthreads();

    // One tile as a stream of MFMAs, each in a fenced packet with its share of the vector work and
    // its operand read from LDS two packets ahead: S and dP of half 0, S and dP of half 1 with half
    // 0's P and dS forming, the updates of half 0 with half 1's, the updates of half 1.
    auto stream = [&](auto bufc) {
      constexpr int buf = decltype(bufc)::value;
      constexpr int kC = Sh::kChunks, kMb = Sh::kDBlocks, kAhead = 2;
      constexpr int kHalf = 2 * kC, kAcc = 4 * kMb, kN = 2 * kHalf + 2 * kAcc, kPerC2 = kAcc / 2;
      f32x16 sc[2], dp[2];
      bf16x8 pb[2][2], db[2][2];
      f32x4 l4[2][4];
      float t0, t1, y0, y1;
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
            if (op == 0) t0 = __builtin_fmaf(sc[hh][e], a.c, -l4[hh][2 * c2 + u][jj]);
            if (op == 1) t1 = __builtin_fmaf(sc[hh][e + 1], a.c, -l4[hh][2 * c2 + u][jj + 1]);
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
    // A tile in which some rows may come before the keys (`lim`: the first row that attends to this
    // lane's key), half after half. The column's query blocks come in ascending order, so such tiles
    // come first, in a loop of their own: beside the stream, in one loop, this would cost the stream
    // its registers (374 bytes of scratch at d = 96).
    [[maybe_unused]] auto masked = [&](const uint16_t* tq, const uint16_t* tg, const float* tl, const float* td, int lim) {
#pragma unroll 1
      for (int hh = 0; hh < 2; ++hh) {
        f32x16 s = f32x16{}, dp;
        f32x4 l4[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(td + 32 * hh + 8 * u + 4 * hf);
          l4[u] = *reinterpret_cast<const f32x4*>(tl + 32 * hh + 8 * u + 4 * hf);
#pragma unroll
          for (int e = 0; e < 4; ++e) dp[4 * u + e] = d4[e];
        }
#pragma unroll
        for (int cc = 0; cc < Sh::kChunks; ++cc) {
          s = mfma32(rows_frag<D>(tq, ra, hh, cc), kf[cc], s);
          dp = mfma32(rows_frag<D>(tg, ra, hh, cc), vf[cc], dp);
        }
        bf16x8 pb[2], db[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int rr = 32 * hh + 8 * (e / 4) + 4 * hf + e % 4;
          const float p = rr < lim ? 0.f : prob(s[e], a.c, l4[e / 4][e % 4]);
          pb[e / 8][e % 8] = (__bf16)p;
          db[e / 8][e % 8] = (__bf16)(p * dp[e]);
        }
#pragma unroll
        for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
          for (int mb = 0; mb < Sh::kDBlocks; ++mb) {
            dv[mb] = mfma32(cols_frag<D>(tg, ca, mb, 2 * hh + c2), pb[c2], dv[mb]);
            dk[mb] = mfma32(cols_frag<D>(tq, ca, mb, 2 * hh + c2), db[c2], dk[mb]);
          }
      }
    };
    bool more = true;  // a tile is loaded
    if constexpr (CAUSAL) {
      int buf = 0;
      const int own_last = j * kBlock + kBlock - 1;
      while (more && (g.off + block * kBlock < own_last || buf)) {
        more = !nxt.done();
        if (more) load_tile(nxt, buf ^ 1);
        if (wave_active) masked(sQ[buf], sG[buf], sL[buf], sD[buf], key - first);
        if (more) {
          first = nxt.first();
          block = nxt.walk.at;
          nxt.next();
        }
        wait_tile_loads();
        __syncthreads();
        buf ^= 1;
      }
    }
    auto tile_step = [&](auto bufc) {
      constexpr int buf = decltype(bufc)::value;
      more = !nxt.done();
      if (more) load_tile(nxt, buf ^ 1);
      if (wave_active) stream(bufc);
      if (more) nxt.next();
      wait_tile_loads();
      __syncthreads();
    };
    while (more) {
      tile_step(std::integral_constant<int, 0>{});
      if (!more) break;
      tile_step(std::integral_constant<int, 1>{});
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

// Both passes in one launch (two workgroups a compute unit): the key side's items first, they are
// the longer ones, then the query side's units, which fill the places as they fall free.
template <int D, bool CAUSAL>
__global__ __launch_bounds__(kThreadsB, 2) void block_grad_kernel(const BlockBwdArgs a, uint32_t key_wgs) {
  __shared__ uint16_t s0[2][BlockShape<D>::kTileElems], s1[2][BlockShape<D>::kTileElems];
  __shared__ float sL[2][kBlockK], sD[2][kBlockK];
  __shared__ uint32_t bits[kBlockWords];
  if (blockIdx.x < key_wgs) dkdv_unit<D, CAUSAL>(a, blockIdx.x, s0, s1, sL, sD, bits);
  else dq_unit<D>(a, blockIdx.x - key_wgs, s0, s1, bits);
}

// d = 128: the key side's accumulators and operands take 256 registers by themselves, so it runs one
// workgroup a compute unit, and each pass has a launch of its own.
template <int D, bool CAUSAL>
__global__ __launch_bounds__(kThreadsB, 1) void block_dkdv_kernel(const BlockBwdArgs a) {
  __shared__ uint16_t s0[2][BlockShape<D>::kTileElems], s1[2][BlockShape<D>::kTileElems];
  __shared__ float sL[2][kBlockK], sD[2][kBlockK];
  __shared__ uint32_t bits[kBlockWords];
  dkdv_unit<D, CAUSAL>(a, blockIdx.x, s0, s1, sL, sD, bits);
}
template <int D>
__global__ __launch_bounds__(kThreadsB, 2) void block_dq_kernel(const BlockBwdArgs a) {
  __shared__ uint16_t s0[2][BlockShape<D>::kTileElems], s1[2][BlockShape<D>::kTileElems];
  __shared__ uint32_t bits[kBlockWords];
  dq_unit<D>(a, blockIdx.x, s0, s1, bits);
}

// Adds the pieces of a dq unit, in order; a thread takes 4 consecutive d of a row.
template <int D>
__device__ __forceinline__ void sum_dq(const BlockBwdArgs& a, uint32_t lu) {
  const BlockGeo& g = a.g;
  const uint32_t list = lu / a.units;
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

// Adds the pieces of a cut key block, in order: dk, or dv.
template <int D>
__device__ __forceinline__ void sum_dkdv(const BlockBwdArgs& a, uint32_t col, int which) {
  const BlockGeo& g = a.g;
  const int pieces = a.plan[4 * (size_t)col + 1];
  if (pieces == 1) return;
  const int slot = a.plan[4 * (size_t)col + 2];
  if (slot + pieces > a.slots) return;
  const int j = (int)(col % g.nb);
  const size_t row0 = (size_t)(col / g.nb) * g.Skv + (size_t)j * kBlock;
  const int n_rows = min(kBlock, g.Skv - j * kBlock);
  const float* part = a.part_k + ((size_t)slot * 2 + which) * kBlock * D;
  uint16_t* out = which ? a.dv : a.dk;
  for (int x = threadIdx.x; x < n_rows * (D / 4); x += kThreadsB) {
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < pieces; ++p) y += *reinterpret_cast<const f32x4*>(part + (size_t)p * 2 * kBlock * D + 4 * x);
    *reinterpret_cast<u32x2*>(out + row0 * D + 4 * x) = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
  }
}

template <int D>
__global__ __launch_bounds__(kThreadsB) void block_sum_kernel(const BlockBwdArgs a, uint32_t dq_wgs) {
  if (blockIdx.x < dq_wgs) sum_dq<D>(a, blockIdx.x);
  else sum_dkdv<D>(a, (blockIdx.x - dq_wgs) / 2, (blockIdx.x - dq_wgs) % 2);
}

template <int D>
hipError_t block_bwd_for(const BlockBwdArgs& a, hipStream_t s) {
  const BlockGeo& g = a.g;
  const int64_t rows = (int64_t)g.B * g.H * g.Sq;
  const uint32_t cols = (uint32_t)((int64_t)g.B * g.Hkv * g.nb), per = (cols + 7) / 8;
  const uint32_t lists = (uint32_t)((int64_t)g.B * g.Hkv * g.nq);
  const uint32_t prep = (uint32_t)((rows + kPrepRowsB - 1) / kPrepRowsB);
  const uint32_t words = (uint32_t)((int64_t)g.B * g.Hkv * ((g.nq + 31) / 32));
  const size_t lds = std::max((size_t)kPrepRowsB * (D / 8), (size_t)g.nb) * 4;
  block_prep_kernel<D><<<prep + words, kThreadsB, lds, s>>>(a, rows, prep);
  block_plan_kernel<<<8, kPlanThreads, 0, s>>>(a, cols, per);
  const uint32_t keys = 8 * per * (uint32_t)a.pieces_k, queries = xcd_grid(lists * a.units * a.pieces_q);
  if constexpr (D == 128) {
    if (g.causal) block_dkdv_kernel<D, true><<<keys, kThreadsB, 0, s>>>(a);
    else block_dkdv_kernel<D, false><<<keys, kThreadsB, 0, s>>>(a);
    block_dq_kernel<D><<<queries, kThreadsB, 0, s>>>(a);
  } else {
    if (g.causal) block_grad_kernel<D, true><<<keys + queries, kThreadsB, 0, s>>>(a, keys);
    else block_grad_kernel<D, false><<<keys + queries, kThreadsB, 0, s>>>(a, keys);
  }
  const uint32_t sum_q = a.pieces_q > 1 ? lists * a.units : 0, sum_k = a.pieces_k > 1 ? 2 * cols : 0;
  if (sum_q + sum_k) block_sum_kernel<D><<<sum_q + sum_k, kThreadsB, 0, s>>>(a, sum_q);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_bwd(const BlockBwdArgs& a, hipStream_t stream) {
  if (a.g.d == 64) return block_bwd_for<64>(a, stream);
  if (a.g.d == 96) return block_bwd_for<96>(a, stream);
  return block_bwd_for<128>(a, stream);
}

}  // namespace ta
