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
//   plan     deals the columns out to the XCDs by work, cuts long ones (a block that every query
//            keeps) into pieces of at most `entries` query blocks, and orders the pieces longest first;
//            at d = 128 (and enough work) instead one line of all columns, cut into even stretches.
//   dq       one workgroup per unit of 128 query rows, over its list's key tiles:
//            S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T; a lane owns one query.
//   dk, dv   one workgroup per piece of a key block (128 keys, 4 waves of 32), over the 64-row
//            tiles of its query blocks and heads: S = Q K^T, dP = dO V^T, dV^T += dO^T P,
//            dK^T += Q^T dS; a lane owns one key.
//   sum      adds the pieces of cut units, in order.
// Measured, a call, from card to card: 24 heads of 28800 tokens, 32 of 225 blocks each, d = 96: 3440 to 3580
// us, 790 to 760 TFLOP/s as five products and 1105 to 1065 as the seven that run (a library product of
// 16384^3: 1312; vector issue beside the matrix cores). 16 heads on 4 key heads, 16384 tokens, 24 blocks,
// causal, d = 128: 1180 to 1240 us; kernel by kernel dk, dv 700, dq 520, prep 22, sum 16, plan 7. 12 heads of
// 2251 tokens, 6 blocks, d = 64: 46 us, of it 38 for both passes, whose columns and units are few, and two
// short launches around them.
// Roundings: P and dS to bf16 before they enter a product (the matrix cores take fp32 at a sixteenth of
// the rate), and the results at the end; S, dP, delta, all sums and cut pieces' parts are fp32. They
// move the gradients' error against 64 bits, the results' own rounding in it, from 1.8e-3 to 2.4e-3.
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

// Blocks that the rows of query block i may attend to: those below this one.
__device__ __forceinline__ int listable(const BlockGeo& g, int len, int i) {
  const int first = g.off + i * kBlock, last = min(first + min(kBlock, g.Sq - i * kBlock), len) - 1;
  return last < first ? 0 : min(g.nb, (g.causal ? last : len - 1) / kBlock + 1);
}

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
    const int bit = x / g.n_list, j = lists[x];
    if (j >= 0 && j < listable(g, len, i0 + bit)) atomicOr(&col[j], 1u << bit);
  }
  __syncthreads();
  for (int j = threadIdx.x; j < g.nb; j += kThreadsB) a.cols[((size_t)bh * g.nb + j) * words + w] = col[j];
}

// ---------------------------------------------------------------------------------------------
// plan

// One workgroup per XCD. The columns, in order, are dealt out to the XCDs as contiguous shares of
// equal work (a column's query blocks, and a quarter of the mean for its start and end): in causal
// order early blocks have many more query blocks than late ones, and shares of equal count left
// half of the XCDs idle (4 key heads of 128 blocks: 986 us). Each workgroup cuts the columns of its
// share into pieces and lists the pieces longest first (by 64 sizes): popular blocks' pieces start
// the launch, those of blocks that hardly anybody lists even out its end.
// plan[4 col] = the column's query blocks, + 1 = its pieces, + 2 = its first slot; items[xcd * cap
// + i] = {column, piece}; counts[xcd] = items of the share. Items of one size come in any order: when a
// piece runs may differ from call to call, what it adds up and in which order does not.
constexpr int kPlanThreads = 1024, kSizes = 64;

// NT threads; blocks_of(x): the query blocks of column x.
template <int NT, typename Fn>
__device__ __forceinline__ void plan_share(const BlockBwdArgs& a, uint32_t cols, int xcd, Fn&& blocks_of) {
  __shared__ int hist[kSizes];
  __shared__ int64_t wave_sums[NT / 64];
  __shared__ int wave_slots[NT / 64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const uint32_t each = (cols + NT - 1) / NT;
  const uint32_t x0 = min(cols, tid * each), x1 = min(cols, x0 + each);
  auto pieces_of = [&](int n) { return max(1, (n + a.entries - 1) / a.entries); };
  auto slots_of = [&](int pieces) { return pieces > 1 ? pieces : 0; };
  if (tid < kSizes) hist[tid] = 0;
  int64_t own = 0;
  int own_slots = 0;
  for (uint32_t x = x0; x < x1; ++x) {
    const int n = blocks_of(x);
    own += n;
    own_slots += slots_of(pieces_of(n));
  }
  int64_t upto = own;
  int upto_slots = own_slots;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int64_t y = __shfl_up((long long)upto, s);
    const int z = __shfl_up(upto_slots, s);
    if (lane >= s) {
      upto += y;
      upto_slots += z;
    }
  }
  if (lane == 63) {
    wave_sums[wave] = upto;
    wave_slots[wave] = upto_slots;
  }
  __syncthreads();
  int64_t total = 0, before = upto - own;
  int slots_before = upto_slots - own_slots;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wave) {
      before += wave_sums[w];
      slots_before += wave_slots[w];
    }
    total += wave_sums[w];
  }
  const int64_t start = max((int64_t)1, (total + 4 * (int64_t)cols - 1) / (4 * (int64_t)cols));
  const int64_t work = total + start * cols;
  before += start * x0;
  // Entries of pieces of one column differ by at most one: one size stands for all.
  auto size_of = [&](int n, int pieces) {
    return kSizes - 1 - min(kSizes - 1, (int)((int64_t)((n + pieces - 1) / pieces) * kSizes / (a.entries + 1)));
  };
  auto mine = [&](auto&& fn) {
    int64_t at = before;
    int slot = slots_before;
    for (uint32_t x = x0; x < x1; ++x) {
      const int to = (int)(at * 8 / work);
      if (to > xcd) break;
      const int n = blocks_of(x), pieces = pieces_of(n);
      at += n + start;
      if (to == xcd) fn(x, n, pieces, slot);
      slot += slots_of(pieces);
    }
  };
  mine([&](uint32_t x, int n, int pieces, int slot) {
    a.plan[4 * (size_t)x] = n;
    a.plan[4 * (size_t)x + 1] = pieces;
    a.plan[4 * (size_t)x + 2] = pieces > 1 ? slot : 0;
    atomicAdd(&hist[size_of(n, pieces)], pieces);
  });
  __syncthreads();
  if (tid < kSizes) {  // one wave: where each size starts
    const int mine_n = hist[tid];
    int sum = mine_n;
#pragma unroll
    for (int s = 1; s < kSizes; s <<= 1) {
      const int y = __shfl_up(sum, s);
      if (tid >= s) sum += y;
    }
    hist[tid] = sum - mine_n;
    if (tid == kSizes - 1) a.counts[xcd] = min(sum, a.items_cap);
  }
  __syncthreads();
  int2* items = reinterpret_cast<int2*>(a.items) + (size_t)xcd * a.items_cap;
  mine([&](uint32_t x, int n, int pieces, int) {
    const int at = atomicAdd(&hist[size_of(n, pieces)], pieces);
    for (int p = 0; p < pieces; ++p)
      if (at + p < a.items_cap) items[at + p] = int2{(int)x, p};
  });
}

__global__ __launch_bounds__(kPlanThreads) void block_plan_kernel(const BlockBwdArgs a, uint32_t cols) {
  const int words = query_words(a.g);
  plan_share<kPlanThreads>(a, cols, (int)blockIdx.x, [&](uint32_t x) {
    int n = 0;
#pragma unroll 4
    for (int w = 0; w < words; ++w) n += __builtin_popcount(a.cols[(size_t)x * words + w]);
    return n;
  });
}

// Short lists: the plan in the prep launch (2 heads of 500 tokens 21.9 us and 19.3, 12 of 2251 48.9 and
// 47.6). Every one of the eight workgroups turns all lists round in
// its own LDS (a.plan_in_prep: few words and entries), writes its part of the columns and plans its share.
__device__ __forceinline__ void plan_lists(const BlockBwdArgs& a, int xcd, uint32_t* col) {
  const BlockGeo& g = a.g;
  const int words = query_words(g);
  const uint32_t cols = (uint32_t)g.B * g.Hkv * g.nb, all = cols * words;
  for (uint32_t x = threadIdx.x; x < all; x += kThreadsB) col[x] = 0;
  __syncthreads();
  const uint32_t entries = (uint32_t)g.B * g.Hkv * g.nq * g.n_list;
  for (uint32_t x = threadIdx.x; x < entries; x += kThreadsB) {
    const uint32_t list = x / g.n_list, bh = list / g.nq;
    const int i = (int)(list - bh * g.nq), j = a.lists[x];
    const int len = g.lens ? min(max(g.lens[bh / g.Hkv], 0), g.Skv) : g.Skv;
    if (j >= 0 && j < listable(g, len, i)) atomicOr(&col[(bh * g.nb + j) * words + i / 32], 1u << (i % 32));
  }
  __syncthreads();
  for (uint32_t x = xcd * kThreadsB + threadIdx.x; x < all; x += 8 * kThreadsB) a.cols[x] = col[x];
  plan_share<kThreadsB>(a, cols, xcd, [&](uint32_t x) {
    int n = 0;
    for (int w = 0; w < words; ++w) n += __builtin_popcount(col[x * words + w]);
    return n;
  });
}

// ---------------------------------------------------------------------------------------------
// prep's launch, and the plan of the line

template <int D>
__global__ __launch_bounds__(kThreadsB) void block_prep_kernel(const BlockBwdArgs a, int64_t n_rows, uint32_t prep_wgs) {
  constexpr int kPieces = D / 8, kPer = kPrepRowsB * kPieces / kThreadsB;
  static_assert(kPrepRowsB * kPieces == kThreadsB * kPer, "whole pieces per thread");
  extern __shared__ float part[];  // the rows' pieces, or the columns' words
  if (blockIdx.x >= prep_wgs) {
    if (a.plan_in_prep) plan_lists(a, (int)(blockIdx.x - prep_wgs), reinterpret_cast<uint32_t*>(part));
    else column_words(a, blockIdx.x - prep_wgs, reinterpret_cast<uint32_t*>(part));
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
    const bool some = l != -INFINITY;
    a.lse2[r] = some ? l * 1.4426950408889634f : INFINITY;
    a.ndelta[r] = l != l ? l : some ? -acc : 0.f;  // NaN, of a row of NaN, passes into dS (and dv: store_key)
  }
}

// The plan at d = 128, where the key side runs one workgroup a compute unit and an item of the plan above
// was a third of what a unit had to do (units were busy 75% of the launch, so 92%; 16 heads on 4, 16384
// tokens, causal: 1270 us and 1210 in all): all columns form one line, a
// column of n query blocks col_start + 4 n long (col_start: what its start and end, and in causal order
// the masked tiles of its first block, take in quarters of a query block), and `workers` workgroups take
// even stretches of it. A column that several share leaves one partial sum each.
// plan[4 col] = the column's query blocks, + 1 = its pieces, + 2 = its first slot, + 3 = its first
// worker; items[w] = {column, place in it} where worker w starts; counts[0] = workers.
struct KeyLine {
  int64_t each, more;  // every worker's part; workers with one more
  __device__ __forceinline__ KeyLine(int64_t total, int workers) : each(total / workers), more(total % workers) {}
  __device__ __forceinline__ int64_t start(int w) const { return w * each + min((int64_t)w, more); }
  __device__ __forceinline__ int worker(int64_t x) const {
    const int64_t y = x - more * (each + 1);
    return (int)(y < 0 ? x / (each + 1) : more + y / each);
  }
};
// The first of a column's n query blocks that lies at `at` or behind it.
__device__ __forceinline__ int line_entry(int at, int col_start, int n) { return min(max((at - col_start + 3) >> 2, 0), n); }

__global__ __launch_bounds__(kPlanThreads) void block_line_kernel(const BlockBwdArgs a, uint32_t cols) {
  __shared__ int64_t wave_sums[kPlanThreads / 64];
  const int words = query_words(a.g);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const uint32_t each = (cols + kPlanThreads - 1) / kPlanThreads;
  const uint32_t x0 = min(cols, tid * each), x1 = min(cols, x0 + each);
  auto blocks_of = [&](uint32_t x) {
    int n = 0;
#pragma unroll 4
    for (int w = 0; w < words; ++w) n += __builtin_popcount(a.cols[(size_t)x * words + w]);
    return n;
  };
  int64_t own = 0;
  for (uint32_t x = x0; x < x1; ++x) own += blocks_of(x);
  int64_t upto = own;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int64_t y = __shfl_up((long long)upto, s);
    if (lane >= s) upto += y;
  }
  if (lane == 63) wave_sums[wave] = upto;
  __syncthreads();
  int64_t total = 0, before = upto - own;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before += wave_sums[w];
    total += wave_sums[w];
  }
  total = 4 * total + (int64_t)a.col_start * cols;
  const int workers = (int)max((int64_t)1, min((int64_t)kLineWorkers, total / (4 * a.entries)));
  const KeyLine line(total, workers);
  int2* starts = reinterpret_cast<int2*>(a.items);
  if (blockIdx.x == 0 && tid == 0) {
    a.counts[0] = workers;
    starts[workers] = int2{(int)cols, 0};
  }
  int64_t at = 4 * before + (int64_t)a.col_start * x0;
  for (uint32_t x = x0; x < x1; ++x) {
    const int n = blocks_of(x), length = a.col_start + 4 * n;
    if (x % gridDim.x == blockIdx.x) {
      const int first = line.worker(at + (n ? a.col_start : 0)), last = n ? line.worker(at + length - 4) : first;
      const int pieces = last - first + 1;
      a.plan[4 * (size_t)x] = n;
      a.plan[4 * (size_t)x + 1] = pieces;
      a.plan[4 * (size_t)x + 2] = pieces > 1 ? atomicAdd(&a.counts[8], pieces) : 0;
      a.plan[4 * (size_t)x + 3] = first;
      int w = line.worker(at);
      if (line.start(w) < at) ++w;
      for (; w < workers && line.start(w) < at + length; ++w) starts[w] = int2{(int)x, (int)(line.start(w) - at)};
    }
    at += length;
  }
}

// P = exp2(c s - lse2) clamped to [0, 1] (the exponent is <= 0 up to rounding for kept pairs; the
// clamp keeps rows of zeros past a tile's valid range finite, which then add exactly nothing). The clamp
// is part of the exponential's instruction and makes 0 of NaN; what a row of NaN owes dv, store_key adds.
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
  UnitPlace u;
  if (!u.find(g, id, a.units, a.pieces_q)) return;
  const uint32_t list = u.list, lu = list * a.units + u.unit;
  const int piece = u.piece, unit = u.unit, i = u.i, b = u.b, h = u.h, bh = u.b * g.Hkv + u.h;
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
  // The column's query blocks [e0, e1).
  __device__ __forceinline__ void start(const BlockGeo& g, int length, const uint32_t* bits, int words, int e0, int e1) {
    head = half = 0;
    G = g.G;
    off = g.off;
    Sq = g.Sq;
    len = length;
    walk.start(bits, words, e0, e1 - e0);
  }
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

// dK, dV += a 64-row tile in which some rows may come before the keys (`lim`: the first row that
// attends to this lane's key), half after half. The columns' query blocks come in ascending order, so
// such tiles come first, in a loop of their own: beside the unmasked stream, in one loop, this
// would cost the stream its registers (374 bytes of scratch at d = 96).
template <int D>
__device__ __forceinline__ void masked_tile(const uint16_t* tq, const uint16_t* tg, const float* tl, const float* td,
                                            int lim, float c, int hf, const RowsAt<D>& ra, const ColsAt<D>& ca,
                                            const bf16x8 (&kf)[D / 16], const bf16x8 (&vf)[D / 16],
                                            f32x16 (&dk)[D / 32], f32x16 (&dv)[D / 32]) {
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
    for (int cc = 0; cc < D / 16; ++cc) {
      s = mfma32(rows_frag<D>(tq, ra, hh, cc), kf[cc], s);
      dp = mfma32(rows_frag<D>(tg, ra, hh, cc), vf[cc], dp);
    }
    bf16x8 pb[2], db[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int rr = 32 * hh + 8 * (e / 4) + 4 * hf + e % 4;
      const float p = rr < lim ? 0.f : prob(s[e], c, l4[e / 4][e % 4]);
      pb[e / 8][e % 8] = (__bf16)p;
      db[e / 8][e % 8] = (__bf16)(p * dp[e]);
    }
#pragma unroll
    for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb) {
        dv[mb] = mfma32(cols_frag<D>(tg, ca, mb, 2 * hh + c2), pb[c2], dv[mb]);
        dk[mb] = mfma32(cols_frag<D>(tq, ca, mb, 2 * hh + c2), db[c2], dk[mb]);
      }
  }
}

// A piece of a column as one workgroup finds it.
struct KeyPiece {
  uint32_t col;
  int piece, pieces, all;  // all: query blocks of the column
  int j, bh, b, h, len;
  size_t group_row;        // row of the group's first head in [B, H, Sq]
  int e0, e1;              // the piece's query blocks: these of the column's, in order
  // Every XCD runs the items of its share in the plan's order; false past their end.
  __device__ __forceinline__ bool find(const BlockBwdArgs& a, uint32_t id) {
    if (id / 8 >= (uint32_t)a.counts[id % 8]) return false;
    const int2 item = reinterpret_cast<const int2*>(a.items)[(size_t)(id % 8) * a.items_cap + id / 8];
    // The same in every lane; in scalar registers the tiles' addresses are scalar work.
    place(a, (uint32_t)__builtin_amdgcn_readfirstlane(item.x));
    piece = __builtin_amdgcn_readfirstlane(item.y);
    e0 = (int)((int64_t)all * piece / pieces);
    e1 = (int)((int64_t)all * (piece + 1) / pieces);
    return true;
  }
  __device__ __forceinline__ void place(const BlockBwdArgs& a, uint32_t column) {
    const BlockGeo& g = a.g;
    col = column;
    all = __builtin_amdgcn_readfirstlane(a.plan[4 * (size_t)col]);
    pieces = __builtin_amdgcn_readfirstlane(a.plan[4 * (size_t)col + 1]);
    j = (int)(col % g.nb);
    bh = (int)(col / g.nb);
    b = bh / g.Hkv;
    h = bh - b * g.Hkv;
    len = seq_len(g, b);
    group_row = ((size_t)b * g.H + (size_t)h * g.G) * g.Sq;
  }
  __device__ __forceinline__ void load_bits(const BlockBwdArgs& a, uint32_t* bits, int words) const {
    for (int x = threadIdx.x; x < words; x += kThreadsB) bits[x] = a.cols[(size_t)col * words + x];
    __syncthreads();
  }
};

// A lane id the compiler cannot hoist: rows derived from it hold no register across the stream.
__device__ __forceinline__ int fresh_lane() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

// The last position of a row of NaN (its log-sum-exp is NaN) among the piece's query blocks, or -1.
__device__ __forceinline__ int last_nan_row(const BlockBwdArgs& a, const KeyPiece& kp, const uint32_t* bits) {
  const BlockGeo& g = a.g;
  const int lane = fresh_lane();
  int last = -1;
  BitWalk walk;
#pragma unroll 1
  for (walk.start(bits, query_words(g), kp.e0, kp.e1 - kp.e0); walk.at >= 0; walk.next()) {
    const int i0 = walk.at * kBlock, n = min(min(kBlock, g.Sq - i0), kp.len - g.off - i0);
#pragma unroll 1
    for (int head = 0; head < g.G; ++head)
#pragma unroll 1
      for (int t = lane; t < n; t += 64) {
        const float l = a.lse2[kp.group_row + (size_t)head * g.Sq + i0 + t];
        if (l != l) last = max(last, g.off + i0 + t);
      }
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) last = max(last, __shfl_xor(last, s));
  return last;
}

// Stores this lane's key row of dK and dV, or the piece's part of it. Rows of padding are zeros:
// what formed for their zero K and V rows counts for nobody. A row of NaN has NaN for the weights of
// all keys it attends to, which the clamp of P took for 0: dS was NaN all the same, so where a key's
// dK is, such rows are looked for, and dV of the keys up to the last of them (in causal order; else of
// all) is NaN. (Without one the price is a comparison a unit; keeping NaN in P would take an
// instruction a score.)
template <int D, bool CAUSAL>
__device__ __forceinline__ void store_key(const BlockBwdArgs& a, const KeyPiece& kp, const uint32_t* bits, int row, int hf,
                                          f32x16 (&dk)[D / 32], f32x16 (&dv)[D / 32]) {
  const int key = kp.j * kBlock + row;
  if (__builtin_amdgcn_ballot_w64(dk[0][0] != dk[0][0]) != 0) {
    const int last = last_nan_row(a, kp, bits);
    if (last >= (CAUSAL ? key : 0)) {
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
        for (int e = 0; e < 16; ++e) dv[mb][e] = __builtin_nanf("");
    }
  }
  if (key >= kp.len) {
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb) {
      dk[mb] = f32x16{};
      dv[mb] = f32x16{};
    }
  }
  if (kp.pieces == 1) {
    if (key < a.g.Skv) {
      const size_t kr = (size_t)kp.bh * a.g.Skv + key;
      store_bf16<D>(a.dk + kr * D, dk, a.scale, hf);
      store_bf16<D>(a.dv + kr * D, dv, 1.f, hf);
    }
  } else {
    const int slot = a.plan[4 * (size_t)kp.col + 2] + kp.piece;
    if (slot < a.slots) {
      float* part = a.part_k + ((size_t)slot * 2 * kBlock + row) * D;
      store_f32<D>(part, dk, a.scale, hf);
      store_f32<D>(part + (size_t)kBlock * D, dv, 1.f, hf);
    }
  }
}

// The key-side pass of one piece of a key block (d = 64 and 96); `id` as a workgroup id.
template <int D, bool CAUSAL>
__device__ __forceinline__ void dkdv_unit(const BlockBwdArgs& a, uint32_t id, uint16_t (&sQ)[2][BlockShape<D>::kTileElems],
                                          uint16_t (&sG)[2][BlockShape<D>::kTileElems], float (&sL)[2][kBlockK],
                                          float (&sD)[2][kBlockK], uint32_t (&bits)[kBlockWords]) {
  using Sh = BlockShape<D>;
  const BlockGeo& g = a.g;
  KeyPiece kp;
  if (!kp.find(a, id)) return;
  const size_t group_row = kp.group_row;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = lane & 31, hf = lane >> 5;
  const int words = query_words(g);
  kp.load_bits(a, bits, words);

  // This lane's key as the B operand of S = Q K^T and dP = dO V^T.
  const int key = kp.j * kBlock + wave * 32 + n;
  const bool wave_active = kp.j * kBlock + wave * 32 < kp.len;
  const size_t kr = (size_t)kp.bh * g.Skv + key;
  bf16x8 kf[Sh::kChunks], vf[Sh::kChunks];
  lane_row<D>(a.k + kr * D, key < kp.len, a.keep, a.flip, hf, kf);
  lane_row<D>(a.v + kr * D, key < kp.len, ~0u, 0u, hf, vf);
  f32x16 dk[Sh::kDBlocks], dv[Sh::kDBlocks];
#pragma unroll
  for (int mb = 0; mb < Sh::kDBlocks; ++mb) {
    dk[mb] = f32x16{};
    dv[mb] = f32x16{};
  }

  QueryTiles nxt;
  nxt.start(g, kp.len, bits, words, kp.e0, kp.e1);
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
    bool more = true;  // a tile is loaded
    if constexpr (CAUSAL) {
      int buf = 0;
      const int own_last = kp.j * kBlock + kBlock - 1;
      while (more && (g.off + block * kBlock < own_last || buf)) {
        more = !nxt.done();
        if (more) load_tile(nxt, buf ^ 1);
        if (wave_active)
          masked_tile<D>(sQ[buf], sG[buf], sL[buf], sD[buf], key - first, a.c, hf, ra, ca, kf, vf, dk, dv);
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

  store_key<D, CAUSAL>(a, kp, bits, wave * 32 + n, hf, dk, dv);
}

// ---------------------------------------------------------------------------------------------
// dk, dv at d = 128, one wave per SIMD
//
// The accumulators (128 registers), the K and V operands (64) and the scores do not fit 256
// registers, so one 4-wave workgroup runs per compute unit with 512 registers a wave: accumulators in
// AGPRs, what the vector ALU touches in VGPRs. Nothing else on the SIMD hides a stall, so each wave
// runs one unbroken stream of matrix instructions over 32-row query blocks h:
//   S, dP of block h            | P, dS of block h - 1, second half of its rows
//   dV, dK update of h - 1      | P, dS of block h, first half
// with the vector work dealt out a few instructions per MFMA, operands read kAhead packets ahead
// across the phases, and the blocks in a ring of LDS slots, five loaded ahead, so that a barrier every
// two blocks never waits for the block it is about to use. Causal tiles that need a mask come first,
// in the plain form, through the same LDS.

// acc += a b with the accumulator in AGPRs. The compiler does not track an asm MFMA's hazards; none
// arise: a comes from LDS (its wait counts asm operands), b was written by the vector ALU at least
// one MFMA earlier, and acc is read by nothing but these MFMAs, the next on the same accumulator 7
// others later, until the drain after the loop.
__device__ __forceinline__ void mfma_acc(bf16x8 a, bf16x8 b, f32x16& acc) {
  asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}

constexpr int kRing = 8;
constexpr int kRingBlock = 32 * 128;                  // elements of a 32-row block of one tensor
constexpr int kRingSlot = 2 * kRingBlock + 256;       // Q and dO rows, then lse2 and -delta (64 floats each)

template <bool CAUSAL>
__device__ __forceinline__ void dkdv_roll_unit(const BlockBwdArgs& a, const KeyPiece& kp, uint16_t* ring, uint32_t* bits) {
  constexpr int D = 128, kC = D / 16, kMb = D / 32;
  constexpr int kLd = kRingBlock * 2 / 2048;          // loads per wave and block (two waves per tensor)
  constexpr int kAhead = 3;
  const BlockGeo& g = a.g;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int words = query_words(g);
  kp.load_bits(a, bits, words);

  bf16x8 kf[kC], vf[kC];
  f32x16 dk[kMb], dv[kMb];
  {
    const int lane = fresh_lane(), key = kp.j * kBlock + wave * 32 + (lane & 31);
    const size_t kr = (size_t)kp.bh * g.Skv + key;
    lane_row<D>(a.k + kr * D, key < kp.len, a.keep, a.flip, lane >> 5, kf);
    lane_row<D>(a.v + kr * D, key < kp.len, ~0u, 0u, lane >> 5, vf);
  }
#pragma unroll
  for (int mb = 0; mb < kMb; ++mb) dk[mb] = dv[mb] = f32x16{};

  QueryTiles tiles;
  tiles.start(g, kp.len, bits, words, kp.e0, kp.e1);
  if constexpr (CAUSAL) {
    // The column's first blocks, up to where every row comes after every key of the block.
    const int own_last = kp.j * kBlock + kBlock - 1;
    if (!tiles.done() && g.off + tiles.walk.at * kBlock < own_last) {
      const int lane = fresh_lane(), hf = lane >> 5, key = kp.j * kBlock + wave * 32 + (lane & 31);
      constexpr int kTileE = kBlockK * D;
      TileLoads<D> ld;
      ld.init(wave, lane);
      RowsAt<D> ra;
      ra.init(lane & 31, hf);
      ColsAt<D> ca;
      ca.init(lane);
      auto at = [&](int bi) { return ring + bi * (2 * kTileE + 256); };
      auto load_tile = [&](int bi) {
        const size_t row0 = tiles.row0(kp.group_row);
        const int nv = tiles.valid();
        ld.load(a.q + row0 * D, nv, at(bi), wave);
        ld.load(a.dout + row0 * D, nv, at(bi) + kTileE, wave);
        if (wave == 0) {
          load_dword_to_lds(buffer_words(a.lse2 + row0, (uint32_t)(nv * 4)), lds_addr(at(bi) + 2 * kTileE), 4 * lane);
          load_dword_to_lds(buffer_words(a.ndelta + row0, (uint32_t)(nv * 4)), lds_addr(at(bi) + 2 * kTileE + 128),
                            4 * lane);
        }
      };
      auto more = [&]() { return !tiles.done() && g.off + tiles.walk.at * kBlock < own_last; };
      load_tile(0);
      int buf = 0;
      for (bool go = true; go; buf ^= 1) {
        const int first = tiles.first();
        tiles.next();
        wait_tile_loads();
        __syncthreads();
        go = more();
        if (go) load_tile(buf ^ 1);  // the buffer that the tile before the barrier used
        const float* rows = reinterpret_cast<const float*>(at(buf) + 2 * kTileE);
        masked_tile<D>(at(buf), at(buf) + kTileE, rows, rows + 64, key - first, a.c, hf, ra, ca, kf, vf, dk, dv);
      }
      __syncthreads();  // the ring takes the buffers over
    }
  }
  // 32-row blocks left: four for every query block and head, fewer for a short last one (the
  // highest bit a column can have).
  int nb = 0;
  if (!tiles.done()) {
    const int rows = min(g.Sq, kp.len - g.off), last = (rows - 1) / kBlock, short_rows = rows - last * kBlock;
    nb = tiles.walk.left * 4;
    if (kp.e1 == kp.all && (bits[last >> 5] >> (last & 31)) & 1) nb -= 4 - (short_rows + 31) / 32;
    nb = __builtin_amdgcn_readfirstlane(nb * g.G);
  }
  if (nb > 0) {
    const int lane = fresh_lane();
    const int hf = lane >> 5;
    RowsAt<D> ra;
    ra.init(lane & 31, hf);
    ColsAt<D> ca;
    ca.init(lane);
    // Waves 0 and 1 load the Q blocks (half a block each) and lse2, waves 2 and 3 dO and -delta;
    // every wave has the same number of loads in flight.
    const bool second = wave >= 2;
    const uint16_t* const src_all = second ? a.dout : a.q;
    const float* const lsrc_all = second ? a.ndelta : a.lse2;
    int off[kLd];
#pragma unroll
    for (int x = 0; x < kLd; ++x) {
      const int q = 64 * ((wave & 1) * kLd + x) + lane;
      const int r = q / (D / 8), ps = q % (D / 8);
      off[x] = (r * D + 8 * (ps ^ swizzle<D>(r))) * 2;
    }
    const uint32_t lds_dst = lds_addr(ring) + (second ? kRingBlock * 2 : 0) + (wave & 1) * kLd * 1024;
    const uint32_t lds_row_dst = lds_addr(ring) + 4 * kRingBlock + (second ? 256 : 0);
    // The block to load next: its rows start at src / lsrc, `left` valid rows remain of its query
    // block and head (0 past the last block: those loads write zeros), at ring byte offset ld_off.
    const uint16_t* src;
    const float* lsrc;
    int left;
    uint32_t ld_off = 0;
    auto at_head = [&]() {
      const size_t row0 = tiles.row0(kp.group_row);
      src = src_all + row0 * D;
      lsrc = lsrc_all + row0;
      left = tiles.valid();
    };
    at_head();
    auto rsrc = [](const void* p, uint32_t bytes) {  // buffer_words of what is scalar already
      const uint64_t x = reinterpret_cast<uint64_t>(p);
      return i32x4{(int)(uint32_t)x, (int)(uint32_t)(x >> 32), (int)bytes, 0x00020000};
    };
    auto load_part = [&](int x) {
      load_to_lds(rsrc(src, (uint32_t)(min(left, 32) * D * 2)), lds_dst + ld_off + 1024u * x, off[x]);
    };
    auto load_rows = [&]() {
      load_dword_to_lds(rsrc(lsrc, (uint32_t)(min(left, 32) * 4)), lds_row_dst + ld_off, 4 * lane);
    };
    auto load_advance = [&]() {
      ld_off = ld_off == (kRing - 1) * kRingSlot * 2 ? 0 : ld_off + kRingSlot * 2;
      src += 32 * D;
      lsrc += 32;
      left -= 32;
      if (left <= 0) {
        left = 0;
        if (!tiles.done()) {
          if (++tiles.head == tiles.G) {
            tiles.head = 0;
            tiles.walk.next();
          }
          if (!tiles.done()) at_head();
        }
      }
    };
    // Zeros in the last slot: the block that the body before block 0's update runs over. (Weights
    // of zero times block 0's own rows would turn an infinite dO into NaN.) Then blocks 0 .. 4 in
    // flight, the zeros and block 0 visible.
    const int left0 = left;
    left = 0;
    ld_off = (kRing - 1) * kRingSlot * 2;
#pragma unroll
    for (int x = 0; x < kLd; ++x) load_part(x);
    load_rows();
    left = left0;
    ld_off = 0;
#pragma unroll
    for (int y = 0; y < 5; ++y) {
      if (y > 0) load_advance();
#pragma unroll
      for (int x = 0; x < kLd; ++x) load_part(x);
      load_rows();
    }
    wait_loads<4 * (kLd + 1)>();
    __syncthreads();

    // By block parity: S and dP - delta, P and dS of the first 16 row entries (rows
    // 16 c2 + 8 u + 4 hf + j are entries 8 c2 + 4 u + j); p1, d1 of the second.
    f32x16 sc[2], dp[2];
    bf16x8 p0[2], d0[2], p1, d1;
    auto row_values = [&](const uint16_t* at, int first, f32x4& lo, f32x4& hi) {
      const float* L = reinterpret_cast<const float*>(at + 2 * kRingBlock) + first + 4 * hf;
      lo = *reinterpret_cast<const f32x4*>(L);
      hi = *reinterpret_cast<const f32x4*>(L + 8);
    };
    // P and dS of entries 8 c2 .. 8 c2 + 7 as 10 steps per pair of entries (an exponential counts
    // two), dealt out evenly to n packets; packet i's share.
    float t0, t1, y0, y1;
    auto vec_share = [&](auto parc, auto c2c, auto ic, auto nc, const f32x4(&l4)[2]) {
      constexpr int par = decltype(parc)::value, c2 = decltype(c2c)::value, i = decltype(ic)::value,
                    n = decltype(nc)::value;
      if constexpr (i >= 0) {
#pragma unroll
        for (int m = i * 40 / n; m < (i + 1) * 40 / n; ++m) {
          const int op = m % 10, e = 8 * c2 + 2 * (m / 10), w = (e % 8) / 2;
          if (op == 0) t0 = __builtin_fmaf(sc[par][e], a.c, -l4[(e % 8) / 4][e % 4]);
          if (op == 1) t1 = __builtin_fmaf(sc[par][e + 1], a.c, -l4[(e % 8) / 4][e % 4 + 1]);
          if (op == 2) t0 = __builtin_amdgcn_fmed3f(fast_exp2(t0), 0.f, 1.f);
          if (op == 4) t1 = __builtin_amdgcn_fmed3f(fast_exp2(t1), 0.f, 1.f);
          if (op == 6) y0 = t0 * dp[par][e];
          if (op == 7) y1 = t1 * dp[par][e + 1];
          if (op >= 8) {
            const f32x2 v = op == 8 ? f32x2{t0, t1} : f32x2{y0, y1};
            bf16x8& dst = op == 8 ? (c2 ? p1 : p0[par]) : (c2 ? d1 : d0[par]);
            u32x4 x = __builtin_bit_cast(u32x4, dst);
            x[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
            dst = __builtin_bit_cast(bf16x8, x);
          }
        }
      }
    };
    constexpr int kNA = 2 * kC, kNU = 4 * kMb;  // MFMAs of the two phases
    auto frag_a = [&](const uint16_t* at, auto ic) -> bf16x8 {
      constexpr int i = decltype(ic)::value;
      return as_bf16x8(load16(at + (i < kC ? ra.get(i) : kRingBlock + ra.get(i - kC))));
    };
    auto frag_u = [&](const uint16_t* at, auto ic) -> bf16x8 {
      constexpr int i = decltype(ic)::value, c2 = i / (2 * kMb), q = i % (2 * kMb);
      return cols_frag<D>(at + (q % 2 ? 0 : kRingBlock), ca, q / 2, c2);
    };
    bf16x8 pf[kAhead];  // the first fragments of the next phase
    uint32_t at_c = 0, at_p = (kRing - 1) * kRingSlot;  // ring offsets (elements) of blocks h and h - 1
    auto body = [&](auto parc) {
      constexpr int par = decltype(parc)::value;
      const uint32_t at_n = at_c == (kRing - 1) * kRingSlot ? 0 : at_c + kRingSlot;
      const uint16_t *tc = ring + at_c, *tp = ring + at_p, *tn = ring + at_n;
      f32x4 l4[2];
      bf16x8 fr[kAhead + 1];
      using ParC = std::integral_constant<int, par>;
      using ParP = std::integral_constant<int, par ^ 1>;
      row_values(tp, 16, l4[0], l4[1]);
#pragma unroll
      for (int x = 0; x < kAhead; ++x) fr[x] = pf[x];
      __builtin_amdgcn_sched_barrier(0);
      static_for<kNA>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        if constexpr (i + kAhead < kNA) fr[(i + kAhead) % (kAhead + 1)] = frag_a(tc, std::integral_constant<int, i + kAhead>{});
        else pf[i + kAhead - kNA] = frag_u(tp, std::integral_constant<int, i + kAhead - kNA>{});
        if constexpr (i == kC - 2) {  // dP starts at the rows' -delta
          f32x4 d4[4];
          row_values(tc, 64, d4[0], d4[1]);
          row_values(tc, 80, d4[2], d4[3]);
#pragma unroll
          for (int e = 0; e < 16; ++e) dp[par][e] = d4[e / 4][e % 4];
        }
        const bf16x8& f = fr[i % (kAhead + 1)];
        if constexpr (i < kC) sc[par] = mfma32(f, kf[i], i == 0 ? f32x16{} : sc[par]);
        else dp[par] = mfma32(f, vf[i - kC], dp[par]);
        vec_share(ParP{}, std::integral_constant<int, 1>{}, std::integral_constant<int, i - 1>{},
                  std::integral_constant<int, kNA - 1>{}, l4);
        __builtin_amdgcn_sched_barrier(0);
      });
      // Keeps the compiler from sinking the packets' vector work past the branch in load_advance.
      asm volatile("" : "+v"(p1), "+v"(d1));
      load_advance();
      if constexpr (par == 0) {
        // Blocks h + 1 and h + 2 have landed (those of h + 3 and h + 4 may be in flight), for every
        // wave once all are here; every wave is also done with block h - 2, so the slots of blocks
        // h - 3 and h - 2 can take blocks h + 5 and h + 6.
        wait_loads<2 * (kLd + 1)>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      row_values(tc, 0, l4[0], l4[1]);
#pragma unroll
      for (int x = 0; x < kAhead; ++x) fr[x] = pf[x];
      __builtin_amdgcn_sched_barrier(0);
      static_for<kNU>([&](auto ic) {
        constexpr int i = decltype(ic)::value, c2 = i / (2 * kMb), q = i % (2 * kMb), mb = q / 2;
        if constexpr (i + kAhead < kNU) fr[(i + kAhead) % (kAhead + 1)] = frag_u(tp, std::integral_constant<int, i + kAhead>{});
        else pf[i + kAhead - kNU] = frag_a(tn, std::integral_constant<int, i + kAhead - kNU>{});
        if constexpr (i >= 1 && i <= kLd) load_part(i - 1);
        if constexpr (i == kLd + 1) load_rows();
        const bf16x8& f = fr[i % (kAhead + 1)];
        if constexpr (q % 2) mfma_acc(f, c2 ? d1 : d0[par ^ 1], dk[mb]);
        else mfma_acc(f, c2 ? p1 : p0[par ^ 1], dv[mb]);
        vec_share(ParC{}, std::integral_constant<int, 0>{}, std::integral_constant<int, i - 2>{},
                  std::integral_constant<int, kNU - 2>{}, l4);
        __builtin_amdgcn_sched_barrier(0);
      });
      asm volatile("" : "+v"(p0[par]), "+v"(d0[par]));
      at_p = at_c;
      at_c = at_n;
    };
    // Before block 0 there is nothing to update: P, dS (exp2(-inf)) and rows are zero. Blocks nb and
    // nb + 1 are zeros, so the bodies past the last block add exactly nothing.
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      sc[1][e] = -INFINITY;
      dp[1][e] = 0.f;
    }
    p0[1] = d0[1] = as_bf16x8(u32x4{0u, 0u, 0u, 0u});
    static_for<kAhead>([&](auto jc) { pf[decltype(jc)::value] = frag_a(ring, jc); });
    for (int h = 0; h <= nb; h += 2) {
      body(std::integral_constant<int, 0>{});
      body(std::integral_constant<int, 1>{});
    }
    wait_tile_loads();
  }
  // The last MFMAs are done before the accumulators are read (16 passes at most).
#pragma unroll
  for (int mb = 0; mb < kMb; ++mb) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(dk[mb]), "+a"(dv[mb]));
  const int lane = fresh_lane();
  store_key<D, CAUSAL>(a, kp, bits, wave * 32 + (lane & 31), lane >> 5, dk, dv);
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

// d = 128: each pass has a launch of its own, the key side one workgroup a compute unit, each with an item
// of the plan or (a.line) with its stretch of the line of all columns; an XCD's workgroups take
// neighbouring ones.
template <bool CAUSAL>
__global__ __launch_bounds__(kThreadsB, 1) void block_dkdv_kernel(const BlockBwdArgs a, int cols) {
  __shared__ __attribute__((aligned(1024))) uint16_t ring[kRing * kRingSlot];
  __shared__ uint32_t bits[kBlockWords];
  KeyPiece kp;
  int w = 0, first, first_at = 0, last, last_at = 0;
  if (a.line) {
    const int workers = a.counts[0], id = (int)blockIdx.x;
    w = workers == kLineWorkers ? id % 8 * (kLineWorkers / 8) + id / 8 : id;
    if (w >= workers) return;
    const int2* starts = reinterpret_cast<const int2*>(a.items);
    const int2 from = starts[w], to = starts[w + 1];
    first = __builtin_amdgcn_readfirstlane(from.x);
    first_at = __builtin_amdgcn_readfirstlane(from.y);
    last = __builtin_amdgcn_readfirstlane(to.x);
    last_at = __builtin_amdgcn_readfirstlane(to.y);
  } else {
    if (!kp.find(a, blockIdx.x)) return;
    first = last = (int)kp.col;
  }
#pragma unroll 1
  for (int col = first; col <= last && col < cols; ++col) {
    if (a.line) {
      kp.place(a, (uint32_t)col);
      const int at = col == first ? first_at : 0;
      kp.e0 = line_entry(at, a.col_start, kp.all);
      kp.e1 = col == last ? line_entry(last_at, a.col_start, kp.all) : kp.all;
      // A column without query blocks gets its zeros from the workgroup whose stretch holds its start.
      if (kp.all == 0 ? at != 0 || (col == last && last_at == 0) : kp.e0 >= kp.e1) continue;
      kp.piece = w - __builtin_amdgcn_readfirstlane(a.plan[4 * (size_t)col + 3]);
    }
    dkdv_roll_unit<CAUSAL>(a, kp, ring, bits);
    __syncthreads();  // the next column's loads overwrite what slower waves still read
  }
}
template <int D>
__global__ __launch_bounds__(kThreadsB, 2) void block_dq_kernel(const BlockBwdArgs a) {
  __shared__ uint16_t s0[2][BlockShape<D>::kTileElems], s1[2][BlockShape<D>::kTileElems];
  __shared__ uint32_t bits[kBlockWords];
  dq_unit<D>(a, blockIdx.x, s0, s1, bits);
}

// Adds the pieces of 32 rows of a dq unit, in order; a thread takes 4 consecutive d of a row.
template <int D>
__device__ __forceinline__ void sum_dq(const BlockBwdArgs& a, uint32_t lu, int r0) {
  const BlockGeo& g = a.g;
  const uint32_t list = lu / a.units;
  const int unit = (int)(lu % a.units), i = (int)(list % g.nq);
  const int bh = (int)(list / g.nq), b = bh / g.Hkv, h = bh - b * g.Hkv;
  const ListRows rows(g, b, h, i);
  const int n_rows = g.G * rows.tokens;
  const float* part = a.part_q + (size_t)lu * a.pieces_q * kUnitRows * D;
  for (int x = threadIdx.x; x < 32 * (D / 4); x += kThreadsB) {
    const int rr = r0 + x / (D / 4), d0 = 4 * (x % (D / 4)), r = unit * kUnitRows + rr;
    if (r >= n_rows) return;
    int pos;
    const size_t row = rows.global(r, pos);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < a.pieces_q; ++p)
      y += *reinterpret_cast<const f32x4*>(part + ((size_t)p * kUnitRows + rr) * D + d0);
    *reinterpret_cast<u32x2*>(a.dq + row * D + d0) = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
  }
}

// Adds the pieces of 32 rows of a cut key block, in order: dk, or dv.
template <int D>
__device__ __forceinline__ void sum_dkdv(const BlockBwdArgs& a, uint32_t col, int which, int r0) {
  const BlockGeo& g = a.g;
  const int pieces = a.plan[4 * (size_t)col + 1];
  if (pieces == 1) return;
  const int slot = a.plan[4 * (size_t)col + 2];
  if (slot + pieces > a.slots) return;
  const int j = (int)(col % g.nb);
  const size_t row0 = (size_t)(col / g.nb) * g.Skv + (size_t)j * kBlock;
  const int end = min(r0 + 32, min(kBlock, g.Skv - j * kBlock));
  const float* part = a.part_k + ((size_t)slot * 2 + which) * kBlock * D;
  uint16_t* out = which ? a.dv : a.dk;
  for (int x = r0 * (D / 4) + threadIdx.x; x < end * (D / 4); x += kThreadsB) {
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = 0; p < pieces; ++p) y += *reinterpret_cast<const f32x4*>(part + (size_t)p * 2 * kBlock * D + 4 * x);
    *reinterpret_cast<u32x2*>(out + row0 * D + 4 * x) = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
  }
}

template <int D>
__global__ __launch_bounds__(kThreadsB) void block_sum_kernel(const BlockBwdArgs a, uint32_t dq_wgs) {
  if (blockIdx.x < dq_wgs) {
    sum_dq<D>(a, blockIdx.x / 4, blockIdx.x % 4 * 32);
  } else {
    const uint32_t x = blockIdx.x - dq_wgs;
    sum_dkdv<D>(a, x / 8, x % 2, (int)(x % 8 / 2) * 32);
  }
}

template <int D>
hipError_t block_bwd_for(const BlockBwdArgs& a, hipStream_t s) {
  const BlockGeo& g = a.g;
  const int64_t rows = (int64_t)g.B * g.H * g.Sq;
  const uint32_t cols = (uint32_t)((int64_t)g.B * g.Hkv * g.nb);
  const uint32_t lists = (uint32_t)((int64_t)g.B * g.Hkv * g.nq);
  const uint32_t prep = (uint32_t)((rows + kPrepRowsB - 1) / kPrepRowsB);
  const uint32_t words = (uint32_t)((int64_t)g.B * g.Hkv * ((g.nq + 31) / 32));
  const size_t column_lds = a.plan_in_prep ? (size_t)cols * ((g.nq + 31) / 32) : (size_t)g.nb;
  const size_t lds = std::max((size_t)kPrepRowsB * (D / 8), column_lds) * 4;
  block_prep_kernel<D><<<prep + (a.plan_in_prep ? 8 : words), kThreadsB, lds, s>>>(a, rows, prep);
  if (a.line) block_line_kernel<<<8, kPlanThreads, 0, s>>>(a, cols);
  else if (!a.plan_in_prep) block_plan_kernel<<<8, kPlanThreads, 0, s>>>(a, cols);
  const uint32_t keys = a.line ? kLineWorkers : 8 * (uint32_t)a.items_cap, queries = unit_grid(g, a.units * a.pieces_q);
  if constexpr (D == 128) {
    if (g.causal) block_dkdv_kernel<true><<<keys, kThreadsB, 0, s>>>(a, (int)cols);
    else block_dkdv_kernel<false><<<keys, kThreadsB, 0, s>>>(a, (int)cols);
    block_dq_kernel<D><<<queries, kThreadsB, 0, s>>>(a);
  } else {
    if (g.causal) block_grad_kernel<D, true><<<keys + queries, kThreadsB, 0, s>>>(a, keys);
    else block_grad_kernel<D, false><<<keys + queries, kThreadsB, 0, s>>>(a, keys);
  }
  const uint32_t sum_q = a.pieces_q > 1 ? 4 * lists * a.units : 0, sum_k = a.pieces_k > 1 ? 8 * cols : 0;
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
