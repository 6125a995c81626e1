// Device helpers of the block attention kernels: 64-row tiles in LDS and their fragments, rows of
// grouped heads, and bitmaps of blocks.
#pragma once
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "block_launch.h"
#include "tile_common.h"

namespace ta {
namespace {

constexpr int kThreadsB = 256;
constexpr int kWavesB = 4;
constexpr int kUnitRows = 128;  // rows of a unit: 4 waves of 32
constexpr float kNoMax = -1e30f;  // a running maximum (base-2 logits) before the first key

template <int D>
struct BlockShape {
  static constexpr int kChunks = D / 16;
  static constexpr int kDBlocks = D / 32;
  static constexpr int kPieces = D / 8;
  static constexpr int kTileElems = kBlockK * D;
  static constexpr int kLoadsPerWave = kBlockK * kPieces / 64 / kWavesB;
  static_assert(kBlockK * kPieces == 64 * kWavesB * kLoadsPerWave, "whole loads per wave");
};

// LDS layout of a 64-row tile: rows of D / 8 16-byte pieces, piece p of row r at p ^ swizzle(r).
// Every tile is read both by rows (16 bytes a lane, 16 consecutive rows an access) and transposed
// (4 consecutive rows of 64 bytes): the swizzle spreads a piece column of 16 consecutive rows over
// all banks and the 64-byte quads of 4 consecutive rows over different bank groups.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
  if constexpr (D == 64) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  else if constexpr (D == 96) return (r >> 2) & 3;
  else return ((r & 3) << 2) | ((r >> 2) & 3);
}
template <int D>
__device__ __forceinline__ int slot_of(int r, int p) { return (r * (D / 8) + (p ^ swizzle<D>(r))) * 8; }

// Direct global -> LDS loads of one 64-row tile of contiguous rows; rows past n_valid read as zeros.
template <int D>
struct TileLoads {
  int off[BlockShape<D>::kLoadsPerWave];
  __device__ __forceinline__ void init(int wave, int lane) {
#pragma unroll
    for (int j = 0; j < BlockShape<D>::kLoadsPerWave; ++j) {
      const int q = 64 * (wave + kWavesB * j) + lane;
      const int r = q / BlockShape<D>::kPieces, ps = q % BlockShape<D>::kPieces;
      off[j] = (r * D + 8 * (ps ^ swizzle<D>(r))) * 2;
    }
  }
  __device__ __forceinline__ void load(const uint16_t* row0, int n_valid, const uint16_t* lds, int wave) const {
    const i32x4 rs = buffer_words(row0, (uint32_t)(max(n_valid, 0) * D * 2));
    const uint32_t base = lds_addr(lds);
#pragma unroll
    for (int j = 0; j < BlockShape<D>::kLoadsPerWave; ++j)
      load_to_lds(rs, __builtin_amdgcn_readfirstlane(base + 1024u * (uint32_t)(wave + kWavesB * j)), off[j]);
  }
};

// A operand by rows: lane (n, h) reads row n of a 32-row block, piece 2 cc + h of chunk cc.
template <int D>
struct RowsAt {
  static constexpr int kN = D == 96 ? 2 : D / 16;  // at d = 96 chunks cc and cc + 2 lie 4 pieces apart
  int at[kN];
  __device__ __forceinline__ void init(int n, int hf) {
#pragma unroll
    for (int cc = 0; cc < kN; ++cc) at[cc] = slot_of<D>(n, 2 * cc + hf);
  }
  __device__ __forceinline__ int get(int cc) const {
    if constexpr (D == 96) return at[cc & 1] + 32 * (cc >> 1);
    else return at[cc];
  }
};
template <int D>
__device__ __forceinline__ bf16x8 rows_frag(const uint16_t* tile, const RowsAt<D>& ra, int rb, int cc) {
  return as_bf16x8(load16(tile + rb * 32 * D + ra.get(cc)));
}

// A operand transposed (rows = d, contraction over tile rows), by the LDS transpose load: lane l
// (g = l / 16, j = l % 16) reads tile row 4 (g / 2) + j / 4 (and that + 8), d = 32 mb + 16 (g % 2) +
// 4 (j % 4) .. + 3; the contraction index of lane half h is tile rows 16 ch + 4 h + (0..3) and
// 16 ch + 8 + 4 h + (0..3), the order in which a C fragment's entries 8 c2 .. 8 c2 + 7 hold theirs.
template <int D>
struct ColsAt {
  static constexpr int kN = D == 96 ? 1 : D / 32;
  int lo[kN], hi[kN];
  __device__ __forceinline__ void init(int lane) {
    const int g = lane >> 4, j = lane & 15;
    const int r = 4 * (g >> 1) + (j >> 2);
#pragma unroll
    for (int mb = 0; mb < kN; ++mb) {
      const int p = 4 * mb + 2 * (g & 1) + ((j >> 1) & 1);
      lo[mb] = slot_of<D>(r, p) + 4 * (j & 1);
      hi[mb] = slot_of<D>(r + 8, p) + 4 * (j & 1);
    }
  }
  __device__ __forceinline__ int get_lo(int mb) const { return D == 96 ? lo[0] + 32 * mb : lo[mb]; }
  __device__ __forceinline__ int get_hi(int mb) const { return D == 96 ? hi[0] + 32 * mb : hi[mb]; }
};
template <int D>
__device__ __forceinline__ bf16x8 cols_frag(const uint16_t* tile, const ColsAt<D>& ca, int mb, int ch) {
  const uint16_t* p = tile + 16 * ch * D;
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + ca.get_lo(mb)));
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + ca.get_hi(mb)));
  const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
  return as_bf16x8(u32x4{a[0], a[1], b[0], b[1]});
}

// B operand: this lane's row (query or key), d = 16 cc + 8 h .. + 7.
template <int D>
__device__ __forceinline__ void lane_row(const uint16_t* row, bool valid, uint32_t keep, uint32_t flip, int hf,
                                         bf16x8 (&x)[D / 16]) {
#pragma unroll
  for (int cc = 0; cc < D / 16; ++cc) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (valid) w = (load16(row + 16 * cc + 8 * hf) & keep) ^ flip;
    x[cc] = as_bf16x8(w);
  }
}

// Stores this lane's row from a transposed accumulator (entry 4 i + j of block mb holds
// d = 32 mb + 8 i + 4 h + j), times s.
template <int D>
__device__ __forceinline__ void store_bf16(uint16_t* row, const f32x16 (&acc)[D / 32], float s, int hf) {
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 x = {acc[mb][4 * i] * s, acc[mb][4 * i + 1] * s, acc[mb][4 * i + 2] * s, acc[mb][4 * i + 3] * s};
      *reinterpret_cast<u32x2*>(row + 32 * mb + 8 * i + 4 * hf) =
          __builtin_bit_cast(u32x2, __builtin_convertvector(x, bf16x4));
    }
}
template <int D>
__device__ __forceinline__ void store_f32(float* row, const f32x16 (&acc)[D / 32], float s, int hf) {
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 x = {acc[mb][4 * i] * s, acc[mb][4 * i + 1] * s, acc[mb][4 * i + 2] * s, acc[mb][4 * i + 3] * s};
      *reinterpret_cast<f32x4*>(row + 32 * mb + 8 * i + 4 * hf) = x;
    }
}

// Tokens of sequence b (b is the same in every lane).
__device__ __forceinline__ int seq_len(const BlockGeo& g, int b) {
  return g.lens ? __builtin_amdgcn_readfirstlane(min(max(g.lens[b], 0), g.Skv)) : g.Skv;
}

// The rows of one list: the `tokens` query tokens of block i of every head of the group, head after
// head. Full blocks put one head into each 128-row unit; a short last block packs the heads.
struct ListRows {
  int tokens;   // query tokens of the block, padding among them
  int first;    // position of the block's first token
  int len;      // tokens of the sequence
  size_t row0;  // row of head h * G's first token of the block in [B, H, Sq]
  int Sq;
  __device__ __forceinline__ ListRows(const BlockGeo& g, int b, int h, int i) {
    tokens = min(kBlock, g.Sq - i * kBlock);
    first = g.off + i * kBlock;
    len = seq_len(g, b);
    row0 = ((size_t)b * g.H + (size_t)h * g.G) * g.Sq + (size_t)i * kBlock;
    Sq = g.Sq;
  }
  // Row r of the list: its row in [B, H, Sq], and its position.
  __device__ __forceinline__ size_t global(int r, int& pos) const {
    const int head = tokens == kBlock ? r / kBlock : r / tokens, t = r - head * tokens;
    pos = first + t;
    return row0 + (size_t)head * Sq + t;
  }
  // The last position that holds a valid row, or first - 1.
  __device__ __forceinline__ int last() const { return min(first + tokens, len) - 1; }
};

// The unit that a workgroup runs: piece `piece` of the 128 rows `unit` of a list. Workgroup id goes to
// XCD id % 8. Where all lists are alike (no causal order, no lengths) each XCD runs a contiguous
// share of the lists, so that the heads it reads stay in its L2. Else lists differ in length, and
// they are dealt out one by one, late query blocks (causal: the long lists) first; with a multiple
// of 8 key heads over the batch each XCD still sees its own heads only. A list's units stay together.
struct UnitPlace {
  uint32_t list;
  int unit, piece, i, b, h;
  __device__ __forceinline__ bool find(const BlockGeo& g, uint32_t id, int units, int pieces) {
    const uint32_t heads = (uint32_t)g.B * g.Hkv, lists = heads * g.nq, per = (lists + 7) / 8;
    const uint32_t at = id / 8, of = (uint32_t)(units * pieces), l = at / of, rem = at - l * of;
    unit = (int)(rem / pieces);
    piece = (int)(rem - (uint32_t)unit * pieces);
    uint32_t bh;
    if (!g.causal && !g.lens) {
      list = (id % 8) * per + l;
      if (l >= per || list >= lists) return false;
      bh = list / g.nq;
      i = (int)(list - bh * g.nq);
    } else {
      const uint32_t x = l * 8 + id % 8;
      if (x >= lists) return false;
      const uint32_t late = x / heads;
      bh = x - late * heads;
      i = g.nq - 1 - (int)late;
      list = bh * g.nq + i;
    }
    b = (int)(bh / g.Hkv);
    h = (int)(bh - (uint32_t)b * g.Hkv);
    return true;
  }
};
inline uint32_t unit_grid(const BlockGeo& g, int of) {
  return ((uint32_t)((int64_t)g.B * g.Hkv * g.nq) + 7) / 8 * 8 * (uint32_t)of;
}

// A list as a bitmap in LDS (all threads; ends with a barrier): entries that name no block, blocks
// past the sequence's end and (causal) past the last row's position are left out, a block listed
// twice is one bit.
__device__ __forceinline__ void list_bits(const BlockGeo& g, const int32_t* list, const ListRows& rows,
                                          uint32_t* bits, int words) {
  for (int x = threadIdx.x; x < words; x += kThreadsB) bits[x] = 0;
  __syncthreads();
  const int last = rows.last();
  const int end = last < rows.first ? 0 : min(g.nb, ((g.causal ? last : rows.len - 1) / kBlock) + 1);
  for (int x = threadIdx.x; x < g.n_list; x += kThreadsB) {
    const int j = list[x];
    if (j >= 0 && j < end) atomicOr(&bits[j >> 5], 1u << (j & 31));
  }
  __syncthreads();
}

// Walks the set bits of a bitmap in LDS in ascending order; wave-uniform.
struct BitWalk {
  const uint32_t* bits;
  int words, word, at;  // at: the bit, or -1 past the last one
  uint32_t cur;
  int left;             // bits still to come, the current one among them
  // From bit `skip` (counting set bits), `n` bits at most.
  __device__ __forceinline__ void start(const uint32_t* b, int n_words, int skip, int n) {
    bits = b;
    words = n_words;
    left = n;
    word = -1;
    cur = 0;
    while (skip >= 0 && ++word < words) {
      cur = (uint32_t)__builtin_amdgcn_readfirstlane((int)bits[word]);
      const int c = __builtin_popcount(cur);
      if (c > skip) break;
      skip -= c;
      cur = 0;
    }
    for (; skip > 0 && cur; --skip) cur &= cur - 1;
    take();
  }
  __device__ __forceinline__ void take() {
    at = -1;
    if (left <= 0) return;
    while (cur == 0) {
      if (++word >= words) return;
      cur = (uint32_t)__builtin_amdgcn_readfirstlane((int)bits[word]);
    }
    at = 32 * word + __builtin_ctz(cur);
    cur &= cur - 1;
  }
  __device__ __forceinline__ void next() {
    --left;
    take();
  }
};

// Set bits of a bitmap in LDS, the same in every lane.
__device__ __forceinline__ int count_bits(const uint32_t* bits, int words) {
  int n = 0;
  for (int x = threadIdx.x & 63; x < words; x += 64) n += __builtin_popcount(bits[x]);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) n += __shfl_xor(n, s);
  return __builtin_amdgcn_readfirstlane(n);
}

// The 64-token tiles of the listed key blocks: tile `half` of block walk.at, key position key0().
struct KeyTiles {
  BitWalk walk;
  int half;
  int end;  // keys from here on are left out of the walk: the sequence's end, or past the last row
  __device__ __forceinline__ bool done() const { return walk.at < 0; }
  __device__ __forceinline__ int key0() const { return walk.at * kBlock + half * kBlockK; }
  __device__ __forceinline__ void next() {
    if (half == 0 && walk.at * kBlock + kBlockK < end) {
      half = 1;
    } else {
      half = 0;
      walk.next();
    }
  }
};

// Keys of a 32-key block past `lim` (an index into the 64-key tile, per lane) get -inf.
__device__ __forceinline__ void mask_keys(f32x16& s, int kb, int hf, int lim) {
  const int l = lim - 4 * hf - 32 * kb;
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (8 * (r >> 2) + (r & 3) > l) s[r] = -INFINITY;
}

// fn(integral_constant<int, i>) for i = 0 .. N-1, in order.
template <int N, int I = 0, typename Fn>
__device__ __forceinline__ void static_for(Fn&& fn) {
  if constexpr (I < N) {
    fn(std::integral_constant<int, I>{});
    static_for<N, I + 1>(static_cast<Fn&&>(fn));
  }
}

}  // namespace
}  // namespace ta
