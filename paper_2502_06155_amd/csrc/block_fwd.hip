// gfx950 (MI355X, CDNA4) kernel of attention over selected blocks.
//
// Work. A unit is 128 rows of one list: with full query blocks one head's block, 4 waves of 32 rows,
// which share the list and with it every key and value tile. 64-key tiles go from memory straight
// into LDS (two buffers, the next tile lands while one is consumed), and each wave computes
//   S^T = K Q^T (v_mfma_f32_32x32x16_bf16, a lane owns one query and 16 of every 32 keys),
//   weights exp2(c s - m) in base 2, O^T += V^T P^T with V read transposed from LDS.
// The reference m of the exponentials moves only when a lane's sum of weights over 32 keys passes
// 2^10 (the first block of a row always moves it): weights up to that are as exact as weights up
// to 1, and the common path needs no row maximum. Row sums add the weights in fp32 before they are
// rounded to bf16 for the second product, so the log-sum-exp keeps fp32 accuracy. (The matrix cores
// take bf16 at this rate and fp32 at a sixteenth of it; the rounding moves the error against 64 bits,
// the results' own rounding in it, from 1.7e-3 to 1.8e-3.)
//
// What bounds it: vector issue beside the matrix cores, an exponential, a multiply-add, an addition and
// half a conversion a score, and at this size the card's power. 6 heads of 86400 tokens, 68 of 675 blocks
// each, d = 96: 1610 to 1700 us a call from card to card = 1075 to 1020 TFLOP/s of kept pairs, 78 to 82% of
// what a library product of 16384^3 reaches (1312); 1580 on a rested card. Two column blocks of 32 rows a
// wave, which feed two matrix instructions with every operand read (the waves split the keys), took 1690
// where one took 1640: LDS is not the bound.
//
// The list becomes a bitmap in LDS at the start (a few hundred entries): repeated and impossible
// entries vanish, the blocks come in ascending order whatever the list's order was, and the walk
// over them costs a scalar bit scan per block.
//
// Units of one list, and of one (batch, key head) as far as the balance allows (UnitPlace), run on one
// XCD next to each other: the lists of neighbouring query blocks share blocks, and so do the heads
// of a group, which the XCD's L2 then holds. Where units
// are few, each list is cut into pieces by its number of blocks and a second kernel joins the
// pieces' results by their log-sum-exp (8 sequences of one token, 32 of 256 blocks, 4 key heads of 128:
// 15.8 us and 4 for the merge; every byte once would take 13.4 at the rate of a copy).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "block_launch.h"
#include "block_tiles.h"

namespace ta {
namespace {

constexpr float kLazyLog2F = 10.f;

__device__ __forceinline__ float lane_max(const f32x16& s) {
  float mx = fmaxf(s[0], s[1]);
#pragma unroll
  for (int r = 2; r < 16; r += 2) mx = fmaxf(fmaxf(mx, s[r]), s[r + 1]);
  return mx;
}

// Weights exp2(c s - m) of one 32-key block as the B operand of the second product, and this
// lane's sum of them.
__device__ __forceinline__ float weights(const f32x16& s, float c, float m, bf16x8 (&p)[2]) {
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int c2 = 0; c2 < 2; ++c2) {
    f32x8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = fast_exp2(__builtin_fmaf(s[8 * c2 + e], c, -m));
      sum[e & 1] += x[e];
    }
    p[c2] = __builtin_convertvector(x, bf16x8);
  }
  return sum[0] + sum[1];
}

template <int D>
__device__ __forceinline__ void scores(const uint16_t* tile, const bf16x8 (&qf)[D / 16], const RowsAt<D>& ra, int kb,
                                       f32x16& s) {
  s = mfma32(rows_frag<D>(tile, ra, kb, 0), qf[0], f32x16{});
#pragma unroll
  for (int cc = 1; cc < D / 16; ++cc) s = mfma32(rows_frag<D>(tile, ra, kb, cc), qf[cc], s);
}
template <int D>
__device__ __forceinline__ void add_values(const uint16_t* tile, const bf16x8 (&p)[2], const ColsAt<D>& ca, int kb,
                                           f32x16 (&o)[D / 32]) {
#pragma unroll
  for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb) o[mb] = mfma32(cols_frag<D>(tile, ca, mb, 2 * kb + c2), p[c2], o[mb]);
}

// add_values for tiles that may hold infinities or NaN and rows that do not see them: the matrix cores
// would add 0 times those to the rows that mask them. Numbers are added alone, and where a row's
// weights of +inf or NaN (-inf or NaN) sum to more than 0, that infinity: both make a NaN.
template <int D>
__device__ __forceinline__ void add_masked_values(const uint16_t* tile, const bf16x8 (&p)[2], const ColsAt<D>& ca, int kb,
                                                  f32x16 (&o)[D / 32]) {
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb) {
    f32x16 up = {}, down = {};
#pragma unroll
    for (int c2 = 0; c2 < 2; ++c2) {
      const u32x4 w = __builtin_bit_cast(u32x4, cols_frag<D>(tile, ca, mb, 2 * kb + c2));
      u32x4 x = {0u, 0u, 0u, 0u}, u = x, v = x;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = 16 * (e % 2);
        const uint32_t y = w[e / 2] >> at & 0xffffu, size = y & 0x7fffu;
        x[e / 2] |= (size < 0x7f80u ? y : 0u) << at;
        u[e / 2] |= (y == 0x7f80u || size > 0x7f80u ? 0x3f80u : 0u) << at;
        v[e / 2] |= (y == 0xff80u || size > 0x7f80u ? 0x3f80u : 0u) << at;
      }
      o[mb] = mfma32(as_bf16x8(x), p[c2], o[mb]);
      up = mfma32(as_bf16x8(u), p[c2], up);
      down = mfma32(as_bf16x8(v), p[c2], down);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (up[e] > 0.f) o[mb][e] += INFINITY;
      if (down[e] > 0.f) o[mb][e] -= INFINITY;
    }
  }
}

template <int D>
__global__ __launch_bounds__(kThreadsB, 2) void block_fwd_kernel(const BlockFwdArgs a) {
  using Sh = BlockShape<D>;
  __shared__ uint16_t sK[2][Sh::kTileElems], sV[2][Sh::kTileElems];
  __shared__ uint32_t bits[kBlockWords];
  const BlockGeo& g = a.g;
  UnitPlace u;
  if (!u.find(g, blockIdx.x, a.units, a.pieces)) return;
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

  // This lane's query row, its B operand, and the last position it attends to (-1: none).
  const int r = unit * kUnitRows + wave * 32 + n;
  int pos = 0;
  const size_t row = rows.global(min(r, n_rows - 1), pos);
  const bool valid = r < n_rows && pos < rows.len;
  const int last = valid ? (g.causal ? pos : rows.len - 1) : -1;
  bf16x8 qf[Sh::kChunks];
  lane_row<D>(a.q + row * D, valid, a.qmask, a.qflip, hf, qf);

  f32x16 o[Sh::kDBlocks];
#pragma unroll
  for (int mb = 0; mb < Sh::kDBlocks; ++mb) o[mb] = f32x16{};
  float m = kNoMax, l = 0.f;
  const float c = a.c, lazy = exp2f(kLazyLog2F);

  KeyTiles nxt;
  nxt.end = g.causal ? min(rows.len, rows.last() + 1) : rows.len;
  auto start = [&]() {
    nxt.half = 0;
    if (a.pieces == 1) {
      nxt.walk.start(bits, words, 0, g.nb);
    } else {
      const int all = count_bits(bits, words);
      const int e0 = (int)((int64_t)all * piece / a.pieces), e1 = (int)((int64_t)all * (piece + 1) / a.pieces);
      nxt.walk.start(bits, words, e0, e1 - e0);
    }
  };
  start();
  if (!nxt.done()) {
    const uint16_t* Kh = a.k + (size_t)bh * g.Skv * D;
    const uint16_t* Vh = a.v + (size_t)bh * g.Skv * D;
    TileLoads<D> ld;
    ld.init(wave, lane);
    RowsAt<D> ra;
    ra.init(n, hf);
    ColsAt<D> ca;
    ca.init(lane);
    ld.load(Kh + (size_t)nxt.key0() * D, rows.len - nxt.key0(), sK[0], wave);
    ld.load(Vh + (size_t)nxt.key0() * D, rows.len - nxt.key0(), sV[0], wave);
    int key0 = nxt.key0();
    nxt.next();
    wait_tile_loads();
    __syncthreads();

    // The weights of a block count once neither of a row's two lanes has a sum above 2^10; otherwise
    // the row's reference is raised to the block's maximum, what is there is rescaled, and the
    // weights form anew. Rows that need not move keep their reference: a row's bits do not depend
    // on the rows beside it.
    auto settle = [&](const f32x16& s, bf16x8(&p)[2], float sum) {
      if (__builtin_amdgcn_ballot_w64(!(sum <= lazy)) != 0) {
        const bool moves = pair_max(sum <= lazy ? 0.f : 1.f) > 0.f;
        const float m_new = moves ? fmaxf(m, pair_max(lane_max(s)) * c) : m;
        const float alpha = fast_exp2(m - m_new);
        l *= alpha;
#pragma unroll
        for (int mb = 0; mb < Sh::kDBlocks; ++mb) o[mb] *= alpha;
        m = m_new;
        sum = weights(s, c, m, p);
      }
      l += sum;
    };
    auto tile_step = [&](auto bufc, bool more) {
      constexpr int buf = decltype(bufc)::value;
      if (more) {
        ld.load(Kh + (size_t)nxt.key0() * D, rows.len - nxt.key0(), sK[buf ^ 1], wave);
        ld.load(Vh + (size_t)nxt.key0() * D, rows.len - nxt.key0(), sV[buf ^ 1], wave);
      }
      const int lim = last - key0;  // the last key of the tile this lane's row attends to
      if (__builtin_amdgcn_ballot_w64(lim >= 0) != 0) {
        const bool mask = __builtin_amdgcn_ballot_w64(lim < kBlockK - 1) != 0;
        f32x16 s0, s1;
        bf16x8 p0[2], p1[2];
        constexpr int kMfma = D / 16, kValu = 48 * 16 / D;
        scores<D>(sK[buf], qf, ra, 0, s0);
        if (mask) mask_keys(s0, 0, hf, lim);
        __builtin_amdgcn_sched_barrier(0);
        scores<D>(sK[buf], qf, ra, 1, s1);
        float sum = weights(s0, c, m, p0);
        spread_valu_over_mfma<kMfma, kValu>();
        settle(s0, p0, sum);
        if (mask) mask_keys(s1, 1, hf, lim);
        __builtin_amdgcn_sched_barrier(0);
        add_values<D>(sV[buf], p0, ca, 0, o);
        sum = weights(s1, c, m, p1);
        spread_valu_over_mfma<kMfma, kValu>();
        settle(s1, p1, sum);
        __builtin_amdgcn_sched_barrier(0);
        add_values<D>(sV[buf], p1, ca, 1, o);
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

    // Sums that are no numbers may come from values that a row masks: then all of it again, with those
    // apart. (Looking for them in the masked tiles beforehand cost 12 to 20% in causal order.)
    float worst = 0.f;
#pragma unroll
    for (int mb = 0; mb < Sh::kDBlocks; ++mb)
#pragma unroll
      for (int e = 0; e < 16; ++e) worst += 0.f * o[mb][e];  // NaN if one of them is an infinity or NaN
    if (__syncthreads_or(worst != worst)) {
      start();
      m = kNoMax;
      l = 0.f;
#pragma unroll
      for (int mb = 0; mb < Sh::kDBlocks; ++mb) o[mb] = f32x16{};
#pragma unroll 1
      for (; !nxt.done(); nxt.next()) {
        key0 = nxt.key0();
        ld.load(Kh + (size_t)key0 * D, rows.len - key0, sK[0], wave);
        ld.load(Vh + (size_t)key0 * D, rows.len - key0, sV[0], wave);
        wait_tile_loads();
        __syncthreads();
        if (__builtin_amdgcn_ballot_w64(last >= key0) != 0) {
#pragma unroll 1
          for (int kb = 0; kb < 2; ++kb) {
            f32x16 s;
            bf16x8 p[2];
            scores<D>(sK[0], qf, ra, kb, s);
            mask_keys(s, kb, hf, last - key0);
            settle(s, p, weights(s, c, m, p));
            add_masked_values<D>(sV[0], p, ca, kb, o);
          }
        }
        __syncthreads();
      }
    }
  }

  l = pair_sum(l);
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const float lse2 = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);  // NaN for a row of NaN
  if (a.pieces > 1) {
    float* part = a.part + (((size_t)lu * a.pieces + piece) * kUnitRows + wave * 32 + n) * (D + 4);
    if (r < n_rows) {
      store_f32<D>(part, o, inv, hf);
      if (hf == 0) part[D] = lse2;
    }
  } else if (r < n_rows) {
    store_bf16<D>(a.out + row * D, o, inv, hf);
    if (a.lse && hf == 0) a.lse[row] = lse2 * 0.69314718055994531f;
  }
}

// Joins the pieces of 16 of a unit's rows, in order; a thread takes 4 consecutive d of a row.
constexpr int kMergeRowsF = 16;

template <int D>
__global__ __launch_bounds__(kThreadsB) void block_merge_kernel(const BlockFwdArgs a) {
  const BlockGeo& g = a.g;
  const uint32_t lu = blockIdx.x, list = lu / a.units;
  const int unit = (int)(lu % a.units), i = (int)(list % g.nq);
  const int bh = (int)(list / g.nq), b = bh / g.Hkv, h = bh - b * g.Hkv;
  const ListRows rows(g, b, h, i);
  const int n_rows = g.G * rows.tokens;
  const float* part = a.part + (size_t)lu * a.pieces * kUnitRows * (D + 4);
  constexpr size_t kStep = (size_t)kUnitRows * (D + 4);
  for (int x = threadIdx.x; x < kMergeRowsF * (D / 4); x += kThreadsB) {
    const int rr = blockIdx.y * kMergeRowsF + x / (D / 4), d0 = 4 * (x % (D / 4)), r = unit * kUnitRows + rr;
    if (r >= n_rows) return;
    int pos;
    const size_t row = rows.global(r, pos);
    const float* p = part + (size_t)rr * (D + 4);
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int y = 0; y < a.pieces; ++y) {
      const f32x4 u = *reinterpret_cast<const f32x4*>(p + y * kStep + d0);
      const float lse2 = p[y * kStep + D], m_new = fmaxf(m, lse2);
      const float f = lse2 == -INFINITY ? 0.f : fast_exp2(lse2 - m_new);  // a NaN stays one
      const float keep = m == -INFINITY ? 0.f : fast_exp2(m - m_new);
      l = l * keep + f;
      o = o * keep + f * u;
      m = m_new;
    }
    if (l > 0.f) o *= 1.f / l;
    *reinterpret_cast<u32x2*>(a.out + row * D + d0) = __builtin_bit_cast(u32x2, __builtin_convertvector(o, bf16x4));
    if (a.lse && d0 == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
  }
}

template <int D>
hipError_t block_fwd_for(const BlockFwdArgs& a, hipStream_t s) {
  const uint32_t units = (uint32_t)a.g.B * a.g.Hkv * a.g.nq * a.units;
  block_fwd_kernel<D><<<unit_grid(a.g, a.units * a.pieces), kThreadsB, 0, s>>>(a);
  if (a.pieces > 1) {
    // Where every unit has few rows (single tokens) only the first of them.
    const int rows = a.g.nq == 1 ? (int)std::min<int64_t>(kUnitRows, (int64_t)a.g.G * a.g.Sq) : kUnitRows;
    block_merge_kernel<D><<<dim3(units, (rows + kMergeRowsF - 1) / kMergeRowsF), kThreadsB, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_fwd(const BlockFwdArgs& a, hipStream_t stream) {
  if (a.g.d == 64) return block_fwd_for<64>(a, stream);
  if (a.g.d == 96) return block_fwd_for<96>(a, stream);
  return block_fwd_for<128>(a, stream);
}

}  // namespace ta
