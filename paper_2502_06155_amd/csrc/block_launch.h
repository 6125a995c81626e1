// Internal interface between the C-ABI host code and the gfx950 kernels of attention over
// selected blocks and over the 8-bit and 4-bit caches.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace ta {

constexpr int kBlock = 128;     // tokens of a block and of a cache page (TA_BLOCK)
constexpr int kBlockWords = 512;  // words of a bitmap over TA_MAX_BLOCKS blocks

// The sizes of one call, shared by all kernels: G = H / Hkv query heads per key head, nq and nb
// query and key blocks, query row r at position off + r.
struct BlockGeo {
  int B, H, Hkv, G, Sq, Skv, off, d, nq, nb, n_list, causal;
  const int32_t* lens;  // [B] or null
};

constexpr int kLineWorkers = 256;  // workgroups of the gradients' key side at d = 128
constexpr int kCacheSegment = 3;  // what a (sequence, head) costs cache attention beside its pages
constexpr int kCache4Segment = 5;  // the same over the 4-bit cache
// Tokens of a head that a workgroup writes to it or reads back: a wave's 64 lanes hold 8 values each.
constexpr int cache4_tokens(int d) { return 4 * (64 / (d / 8)); }

struct MeansArgs {
  const uint16_t* x;
  uint16_t* means;
  int B, H, S, d, nb;
  const int32_t* lens;
};

struct ListsArgs {
  BlockGeo g;
  const uint16_t* q;
  const uint16_t* kmeans;
  int32_t* lists;
  int sink, local;
  int rows;  // query blocks of a workgroup (set by the launch)
};

struct BlockFwdArgs {
  BlockGeo g;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* lists;
  uint16_t* out;
  float* lse;      // or null
  float c;         // > 0: |scale| * log2(e)
  uint32_t qflip;  // 0x80008000 flips the sign of q (negative scale), else 0
  uint32_t qmask;  // 0 zeroes q (scale 0), else ~0
  int units;       // 128-row units per list
  int pieces;      // a unit's list is cut into this many pieces, joined by merge
  float* part;     // pieces > 1: fp32 [list][unit][piece][128][d + 4]: O/l, then the base-2 lse
};

struct BlockBwdArgs {
  BlockGeo g;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* lists;
  const uint16_t* out;
  const uint16_t* dout;
  const float* lse;
  uint16_t* dq;
  uint16_t* dk;
  uint16_t* dv;
  float c, scale;
  uint32_t flip, keep;
  int units;
  int pieces_q;      // pieces of a query unit's list
  int plan_in_prep;  // few list entries: turned round and planned beside prep, not in a launch of its own
  int line;          // the key side takes stretches of the line of all columns, not the plan's items
  int entries;       // query blocks per piece of a key block's column, at most (line: of a stretch, at least)
  int col_start;     // line: what a column costs beside its query blocks, in quarters of one
  int pieces_k;      // pieces of a key block at most
  int slots;         // partial dk, dv blocks there is room for
  float* lse2;       // [B, H, Sq]: base-2 lse, +inf for rows without tokens
  float* ndelta;     // [B, H, Sq]: -<dout, out>
  uint32_t* cols;    // [B, Hkv, nb][nq / 32 words]: the query blocks that list a key block
  int32_t* plan;     // [B, Hkv, nb][4]: entries, pieces, first slot, first worker (line)
  int32_t* counts;   // [9]: items of each XCD's share (line: workers); line: the slot counter
  int32_t* items;    // [8][items_cap][2]: column, piece; line: where each worker starts
  int items_cap;     // items of an XCD's share, at most
  float* part_q;     // pieces_q > 1: fp32 [list][unit][piece][128][d]
  float* part_k;     // fp32 [slot][2][128][d]: dk, dv
};

struct CacheWriteArgs {
  const uint16_t* k;
  const uint16_t* v;
  uint8_t* k_pages;
  uint8_t* v_pages;
  float* k_scales;
  float* v_scales;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* n_new;
  int B, Hkv, N, d, max_pages, n_pages;
};

struct CacheAttnArgs {
  const uint16_t* q;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const float* k_scales;
  const float* v_scales;
  const int32_t* table;
  const int32_t* lens;
  int per_head;
  uint16_t* out;
  float* lse;  // or null
  int B, H, Hkv, G, N, d, max_pages, n_pages;
  float c;     // scale * log2(e)
  int whole;         // a workgroup per (sequence, head) instead of an even share of all pages
  int workers;       // workgroups that share the pages of all sequences
  int row_blocks;    // 32-row (or 16-row) passes over the G * N rows
  float* part;       // fp32 [row block][2 * workers][rows][d + 4]: O/l, base-2 lse
};

struct Cache4WriteArgs {
  const uint16_t* k;
  const uint16_t* v;
  uint8_t* k_pages;
  uint8_t* v_pages;
  uint8_t* k_scales;
  uint8_t* v_scales;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* n_new;  // or null
  uint16_t* k_held;      // or null
  uint16_t* v_held;      // or null
  int B, Hkv, N, d, max_pages, n_pages;
  bool past;  // held values past the caches
};

struct Cache4ReadArgs {
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const uint8_t* k_scales;
  const uint8_t* v_scales;
  const int32_t* table;
  const int32_t* lens;
  uint16_t* k_out;  // or null
  uint16_t* v_out;  // or null
  int B, Hkv, N, d, max_pages, n_pages, first;
  bool past;  // results past the caches
};

// As over the 8-bit cache, with scales of its own (k_scales and v_scales are not looked at).
// c is positive: a scale's sign and its being 0 are in q_flip and q_keep, as in BlockFwdArgs.
struct Cache4AttnArgs : CacheAttnArgs {
  const uint8_t* k_exps;
  const uint8_t* v_exps;
  uint32_t q_flip, q_keep;
  bool eight;  // eight waves a workgroup, one workgroup a compute unit
};

hipError_t launch_block_means(const MeansArgs& a, hipStream_t stream);
hipError_t launch_block_lists(ListsArgs a, hipStream_t stream);
hipError_t launch_block_fwd(const BlockFwdArgs& a, hipStream_t stream);
hipError_t launch_block_bwd(const BlockBwdArgs& a, hipStream_t stream);
hipError_t launch_cache_write(const CacheWriteArgs& a, hipStream_t stream);
hipError_t launch_cache_attn(const CacheAttnArgs& a, hipStream_t stream);
hipError_t launch_cache4_write(const Cache4WriteArgs& a, hipStream_t stream);
hipError_t launch_cache4_read(const Cache4ReadArgs& a, hipStream_t stream);
hipError_t launch_cache4_attn(const Cache4AttnArgs& a, hipStream_t stream);

// Rows of a pass of cache attention over a sequence's G * N rows.
int cache_rows_per_pass(int rows);
int cache4_rows_per_pass(int rows);

}  // namespace ta
