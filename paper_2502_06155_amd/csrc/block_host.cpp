// Host side of the C ABI of attention over selected blocks and over the 8-bit and 4-bit caches: argument
// checks, how work is cut, and the workspaces' sizes. Nothing is allocated and nothing is kept.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <string>

#include "block_attn.h"
#include "block_launch.h"
#include "cache4_attn.h"
#include "host_checks.h"
#include "host_internal.h"

namespace ta {
namespace host {
namespace {

static_assert(kBlock == TA_BLOCK, "block size");
static_assert(kBlockWords * 32 == TA_MAX_BLOCKS, "bitmap size");

int make_geo(BlockGeo& g, int B, int H, int Hkv, int Sq, int Skv, int d, int n_list, int causal, const int32_t* lens) {
  if (B < 1 || H < 1 || Hkv < 1 || Sq < 1 || Skv < 1) return fail(TA_ERR_BAD_SHAPE, "B, H, Hkv, Sq and Skv must be >= 1");
  if (H % Hkv) return fail(TA_ERR_BAD_SHAPE, "H must be a multiple of Hkv");
  if (Sq > Skv) return fail(TA_ERR_BAD_SHAPE, "the query rows are the last Sq of Skv positions: Sq <= Skv");
  if (n_list < 1 || n_list > TA_MAX_BLOCKS) return fail(TA_ERR_BAD_SHAPE, "n_list must be in 1..TA_MAX_BLOCKS");
  if (Skv > TA_MAX_BLOCKS * TA_BLOCK) return fail(TA_ERR_BAD_SHAPE, "Skv exceeds TA_MAX_BLOCKS blocks");
  if (int st = check_dim(d)) return st;
  g.B = B;
  g.H = H;
  g.Hkv = Hkv;
  g.G = H / Hkv;
  g.Sq = Sq;
  g.Skv = Skv;
  g.off = Skv - Sq;
  g.d = d;
  g.nq = (Sq + kBlock - 1) / kBlock;
  g.nb = (Skv + kBlock - 1) / kBlock;
  g.n_list = n_list;
  g.causal = causal != 0;
  g.lens = lens;
  // A workgroup for every query block of a head and for every key block of a key head, at least.
  return check_grid(std::max((double)B * H * g.nq, (double)B * Hkv * g.nb));
}

int64_t lists_of(const BlockGeo& g) { return (int64_t)g.B * g.Hkv * g.nq; }
// 128-row units per list: one per head of full query blocks; a single short block packs its heads.
int units_of(const BlockGeo& g) { return g.nq > 1 ? g.G : (int)(((int64_t)g.G * g.Sq + kBlock - 1) / kBlock); }
// Pieces of every unit's list: enough workgroups for the device, two blocks each at least, where that
// takes four blocks off a workgroup's way (about 2 us a block at most; joining costs 4 us and a launch.
// Forward: 4 blocks in halves 13.7 us, whole 11.6; 6 in halves 25.3 and 18.8. Gradients of 12 heads of
// 2251 tokens, 6 blocks: in halves 49.6, whole 48.8).
constexpr int64_t kPieceWorth = 4;
int pieces_of(const BlockGeo& g) {
  const int64_t units = lists_of(g) * units_of(g);
  const int64_t held = std::min(g.n_list, g.nb);
  const int64_t pieces = std::max<int64_t>(1, std::min(kSlots / units, held / 2));
  return held - (held + pieces - 1) / pieces >= kPieceWorth ? (int)pieces : 1;
}

size_t fwd_bytes(const BlockGeo& g) {
  const int p = pieces_of(g);
  return p == 1 ? 0 : (size_t)(lists_of(g) * units_of(g)) * p * kBlock * (g.d + 4) * sizeof(float);
}

// How the gradient's key side is cut, and where things lie in the workspace.
struct BwdPlan {
  int entries, pieces_q, pieces_k;
  bool line;
  int64_t slots, items_cap;
  size_t off_ndelta, off_cols, off_plan, off_counts, off_items, off_q, off_k, bytes;
};
BwdPlan plan_bwd(const BlockGeo& g) {
  BwdPlan p;
  p.pieces_q = pieces_of(g);
  // Query blocks that all columns hold together, at most, and what a column holds on average. A
  // piece takes up to twice that, or an eighth of a resident workgroup's share of all work where
  // that is more (long launches even out by themselves); in launches of few columns less, so that
  // about one piece per resident workgroup forms, but not below four units of 128 rows. 8 heads of
  // 16384 positions, 24 blocks each, causal, d = 96: 458 us so, 454 at half a piece per workgroup, 472 at
  // two, 517 at four; 6 heads of 8000, 12 blocks, with average columns cut 129, whole (below) 118.
  const int64_t held = lists_of(g) * std::min(g.n_list, g.nb), cols = (int64_t)g.B * g.Hkv * g.nb;
  const int64_t mean = (held + cols - 1) / cols;
  const int64_t most = std::max(2 * mean, held / (8 * kSlots));
  // Where the columns themselves occupy two fifths of the resident workgroups (one a compute unit at
  // d = 128), the average column stays whole. Whole and cut: 216 columns of 6, d = 64 50 and 53 us; 378 of
  // 12, d = 96 118 and 129; 160 of 8, d = 128 82 and 90; below the bound 188 of 20 (six query heads
  // each), d = 64 327 and 272; 144 of 9 41.5 and 38.5.
  const bool enough = 5 * cols >= (g.d == 128 ? kSlots : 2 * kSlots);
  const int64_t least = std::min(most, std::max<int64_t>((3 + g.G) / g.G, enough ? mean : 0));
  p.entries = (int)std::min<int64_t>(INT_MAX, std::min(most, std::max(least, (held + kSlots - 1) / kSlots)));
  p.pieces_k = (g.nq + p.entries - 1) / p.entries;
  // A column in ceil(n / entries) > 1 pieces has n > entries, so fewer than 2 n / entries pieces.
  p.slots = p.pieces_k == 1 ? 0 : std::min(cols * p.pieces_k, 2 * held / p.entries);
  // An XCD's share: with T query blocks in all columns (T <= held) and s = max(1, ceil(T / 4 cols)) the
  // plan counts W = T + s cols of work, and the columns of a share but its last one less than W / 8.
  // So a share has at most W / 8 s <= 5 / 8 cols columns, rounded up, which hold at most
  // W / 8 <= 5 / 32 T + cols / 8 query blocks and those of the last one, nq at most; and a column of n
  // is cut into at most 1 + (n - 1) / entries pieces.
  const int64_t share_blocks = (5 * held + 31) / 32 + (cols + 7) / 8 + g.nq;
  p.items_cap = std::min(cols * p.pieces_k, (5 * cols + 7) / 8 + share_blocks / p.entries);
  // At d = 128 one line of all columns, cut into kLineWorkers stretches at most, of four units of 128 rows
  // at least. Each end of a stretch adds a piece to one column and makes it one of several pieces. (Line
  // and items: 4 key heads of 16384, 24 blocks, causal 1240 and 1335 us; 1 of 7000, 20 blocks 108 and
  // 128. From 6 units a workgroup on: 6 heads of 8000 are 18, 174 and 185; 8 of 2500 are 5, 87 and 86; 16
  // of 1100 are 2, 71 and 65.)
  p.line = g.d == 128 && held * g.G >= 6 * kLineWorkers;
  if (p.line) {
    p.entries = (3 + g.G) / g.G;
    p.pieces_k = g.nq > 1 ? 2 : 1;
    p.slots = g.nq > 1 ? 2 * (kLineWorkers - 1) : 0;
    p.items_cap = kLineWorkers / 8 + 1;
  }
  const size_t rows = (size_t)g.B * g.H * g.Sq;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t at = up(rows * 4);
  p.off_ndelta = at;
  at += up(rows * 4);
  p.off_cols = at;
  at += up((size_t)cols * ((g.nq + 31) / 32) * 4);
  p.off_plan = at;
  at += up((size_t)cols * 16);
  p.off_counts = at;
  at += up(9 * 4);
  p.off_items = at;
  at += up((size_t)p.items_cap * 8 * 8);
  p.off_q = at;
  at += p.pieces_q == 1 ? 0 : up((size_t)(lists_of(g) * units_of(g)) * p.pieces_q * kBlock * g.d * 4);
  p.off_k = at;
  at += up((size_t)p.slots * 2 * kBlock * g.d * 4);
  p.bytes = at;
  return p;
}

// Logits are formed from |scale|; a negative one flips the sign of q (exact in bf16), and 0 zeroes
// q, so that every logit is exactly 0.
void fold_scale(float scale, float& c, uint32_t& flip, uint32_t& keep) {
  c = scale == 0.f ? 1.f : std::max(std::fabs(scale) * 1.4426950408889634f, FLT_MIN);
  flip = scale < 0.f ? 0x80008000u : 0u;
  keep = scale == 0.f ? 0u : ~0u;
}

// Short tables run a workgroup per (sequence, key head), four pages at a time, and need no second
// launch to join parts: up to 8 pages at d = 128 (16 at d = 64), and up to 16 where the segments alone
// fill half of the device. Measured, whole and split: 12 segments of 12 pages at d = 64 8.3 and 9.8 us;
// 8 of 8 at d = 128 12.5 and 10.8 with one launch (3 us of the host's time) less, 8 of 16 19.4 and 11.9;
// 256 of 16 27.5 and 35.1.
bool whole_segments(int64_t segments, int d, int max_pages) {
  return (int64_t)max_pages * d <= 1024 || (max_pages <= 16 && segments >= kSlots / 2);
}

// The workgroups that share a cache attention's pages, and the passes over its rows. Every workgroup of
// every pass may leave two partial results. Up to four passes run all the workgroups that the device
// holds in each; more passes share kPassSlots between them, so that the workspace stays below 70 MB
// whatever N is. One sequence of 32768 tokens, 32 heads on 8 of 128, all workgroups in every pass and
// so: N = 64 144 and 116 us, 69 and 35 MB; 512 1094 and 511, 554 and 35; 2048 4370 and 1864, 2215 and 35.
// A pass of one workgroup has every segment to itself and leaves nothing to join.
constexpr int64_t kPassSlots = 2 * kSlots;
struct CachePlan {
  int workers, passes, rows;
  bool whole, eight;
  size_t bytes;
};
CachePlan plan_cache(int B, int H, int Hkv, int N, int d, int max_pages) {
  CachePlan p;
  const int64_t rows = (int64_t)(H / Hkv) * N;
  p.rows = cache_rows_per_pass((int)std::min<int64_t>(rows, INT_MAX));
  p.passes = (int)((rows + p.rows - 1) / p.rows);
  // Two workgroups run on a compute unit in passes of 16 rows, one in passes of 32.
  p.workers = (int)std::min<int64_t>({p.rows == 16 ? kSlots : kSlots / 2,
                                      p.passes < kPassSlots ? std::max<int64_t>(2, kPassSlots / p.passes) : 1,
                                      (int64_t)B * Hkv * (max_pages + kCacheSegment)});
  p.whole = whole_segments((int64_t)B * Hkv, d, max_pages);
  p.eight = false;
  if (p.whole) p.workers = B * Hkv;
  p.bytes = p.whole || p.workers == 1 ? 0 : (size_t)p.passes * 2 * p.workers * p.rows * (d + 4) * sizeof(float);
  return p;
}
// The 4-bit cache. Passes of 64 and 128 rows share a page's widened codes, and a workgroup of theirs, one a compute unit, takes
// a page at a time, in `page` us, where one of 16 or 32 rows takes four. All passes together have as many workgroups as
// the device holds, at least two each, or one; with 17 to 32 rows half as many for up to four pages each (64 segments of 24 pages, d = 128:
// 18.7 us with 256, 21.4 with 512; 128 of 24, d = 64 18.1 and 16.9; 192 of 157, d = 128 67.5 and 60.7). What a workgroup of
// many rows leaves to join costs `part` us, written and read, so that with P pages sqrt(P page / part) of them are the
// best (64 segments of 16 pages, d = 64, 72 rows: 17.0 us, 18.6 with a fifth fewer), but for few pages, which a workgroup each takes.
// Short tables run a workgroup per segment, in one launch; of eight waves, in passes of 16 rows, where there are more than four
// pages and no more segments than compute units. Alone, a segment takes 5 us and, of 16 rows, 0.22 + 0.002 d us a page
// (0.003 d with four waves); shared, all take 10 us and the bytes' time, d * 1.4e-5 us a page and segment if sequences
// fill half of their tables, or the pages and parts of the workgroups. Up to 24 pages, so that a batch's longest sequence
// costs 14 us at most. Measured, eight waves alone, four alone, and shared, one row: 8 segments of 8 pages at d = 128 8.9, 9.3 and 10.3
// us, of 16 12.7, 14.2 and 10.6; at d = 64 of 12 9.0, 9.7 and 9.7; 64 of 12, d = 128 10.9, 12.5 and 13.3; 128 of 16 14.5, 16.9 and
// 19.7; 256 of 24 22.4, 24.7 and 28.6. Alone and shared, 36 rows: 8 of 2 7.6 and 10.3, of 8 16.7 and 10.9, 64 of 4 11.0 and 15.1, of 16
// 29.6 and 20.9; 120 rows, 8 of 4 16.5 and 15.5, 64 of 4 17.3 and 23.9, 256 of 8 33.1 and 38.8.
struct ManyRows {
  double page, part;
};
ManyRows many_rows(int rows) { return rows == 64 ? ManyRows{1.3, 0.0125} : ManyRows{1.9, 0.025}; }
CachePlan plan_cache4(int B, int H, int Hkv, int N, int d, int max_pages) {
  CachePlan p;
  const int64_t rows = (int64_t)(H / Hkv) * N, segments = (int64_t)B * Hkv;
  p.rows = cache4_rows_per_pass((int)std::min<int64_t>(rows, INT_MAX));
  p.passes = (int)((rows + p.rows - 1) / p.rows);
  const int64_t slots = p.rows > 32 ? kSlots / 2 : kSlots;
  int64_t workers = p.passes < slots ? slots / p.passes : 1;
  const bool eight = p.rows == 16 && max_pages > 4 && segments <= kSlots / 2;
  double alone, shared;
  if (p.rows > 32) {
    const ManyRows m = many_rows(p.rows);
    const double pages = (double)segments * max_pages;
    workers = std::min(workers, std::max<int64_t>(128, (int64_t)std::sqrt(pages * m.page / m.part)));
    alone = m.page * max_pages;
    shared = 2 * std::sqrt(pages * m.page * m.part);
  } else {
    if (p.rows == 32 && segments * max_pages <= 4 * kSlots) workers = kSlots / 2;
    alone = (0.22 + (eight ? 0.002 : 0.003) * d) * max_pages;
    shared = 1.4e-5 * d * (double)segments * max_pages;
  }
  if (p.passes < slots) workers = std::max<int64_t>(2, workers);
  p.workers = (int)std::min(workers, segments * (max_pages + kCache4Segment));
  p.whole = max_pages <= 24 && alone <= 5 + shared;
  p.eight = p.whole && eight;
  if (p.whole) p.workers = (int)segments;
  p.bytes = p.whole || p.workers == 1 ? 0 : (size_t)p.passes * 2 * p.workers * p.rows * (d + 4) * sizeof(float);
  return p;
}
int check_cache(int B, int H, int Hkv, int N, int d, int max_pages, int segment) {
  if (B < 1 || H < 1 || Hkv < 1 || N < 1 || max_pages < 1)
    return fail(TA_ERR_BAD_SHAPE, "B, H, Hkv, N and max_pages must be >= 1");
  if (H % Hkv) return fail(TA_ERR_BAD_SHAPE, "H must be a multiple of Hkv");
  if (max_pages > INT_MAX / TA_BLOCK) return fail(TA_ERR_BAD_SHAPE, "max_pages pages hold more than 2^31 - 1 tokens");
  // The sequences times heads are a grid dimension of their own.
  if ((int64_t)B * Hkv * (max_pages + segment) > INT_MAX)
    return fail(TA_ERR_BAD_SHAPE, "B * Hkv * max_pages exceeds 2^31 - 1");
  if ((int64_t)B * Hkv > 65535) return fail(TA_ERR_BAD_SHAPE, "B * Hkv exceeds the grid limit");
  return check_dim(d);
}
// Attention: so are the passes over its rows and the joins of 8 of them.
int check_cache_attn(int B, int H, int Hkv, int N, int d, int max_pages, int segment) {
  if (int st = check_cache(B, H, Hkv, N, d, max_pages, segment)) return st;
  return (int64_t)(H / Hkv) * N <= 8 * 65535 ? TA_OK : fail(TA_ERR_BAD_SHAPE, "H / Hkv * N exceeds the grid limit");
}

}  // namespace
}  // namespace host
}  // namespace ta

using namespace ta;
using namespace ta::host;

extern "C" {

int block_attn_means(const void* x, void* means, int B, int H, int S, int d, const int32_t* lens, void* stream) {
  if (!x || !means) return fail(TA_ERR_NULL_PTR, "x and means must be non-NULL");
  BlockGeo g;
  if (int st = make_geo(g, B, H, H, S, S, d, 1, 0, lens)) return st;
  if (int st = check_aligned({x, means}, 16, "x and means must be 16-byte aligned")) return st;
  if (int st = check_aligned({lens}, 4, "lens must be 4-byte aligned")) return st;
  const int64_t n = (int64_t)B * H * d;
  if (int st = check_apart({{means, bf16s(n * g.nb)}}, {{x, bf16s(n * S)}, {lens, (size_t)B * 4}})) return st;
  const MeansArgs a{static_cast<const uint16_t*>(x), static_cast<uint16_t*>(means), B, H, S, d, g.nb, lens};
  return launched(launch_block_means(a, static_cast<hipStream_t>(stream)));
}

int block_attn_lists(const void* q, const void* kmeans, int32_t* lists, int B, int H, int Hkv, int Sq, int Skv, int d,
                     int n_list, int sink, int local, int causal, const int32_t* lens, void* stream) {
  if (!q || !kmeans || !lists) return fail(TA_ERR_NULL_PTR, "q, kmeans and lists must be non-NULL");
  ListsArgs a;
  if (int st = make_geo(a.g, B, H, Hkv, Sq, Skv, d, n_list, causal, lens)) return st;
  if (sink < 0 || local < 0) return fail(TA_ERR_BAD_SHAPE, "sink and local must be >= 0");
  // A query block's rows lie in one key block, or in two where the two are cut differently.
  const int64_t own = a.g.off % TA_BLOCK ? 2 : 1;
  const int64_t near = local ? own + (int64_t)(local - 1) * (causal ? 1 : 2) : 0;
  if (std::min<int64_t>((int64_t)sink + near, a.g.nb) > n_list)
    return fail(TA_ERR_BAD_SHAPE, "n_list is smaller than the number of forced blocks");
  if (int st = check_aligned({q, kmeans}, 16, "q and kmeans must be 16-byte aligned")) return st;
  if (int st = check_aligned({lists, lens}, 4, "lists and lens must be 4-byte aligned")) return st;
  if (int st = check_apart({{lists, (size_t)lists_of(a.g) * n_list * 4}},
                           {{q, bf16s((int64_t)B * H * Sq * d)},
                            {kmeans, bf16s((int64_t)B * Hkv * a.g.nb * d)},
                            {lens, (size_t)B * 4}}))
    return st;
  a.q = static_cast<const uint16_t*>(q);
  a.kmeans = static_cast<const uint16_t*>(kmeans);
  a.lists = lists;
  a.sink = sink;
  a.local = local;
  return launched(launch_block_lists(a, static_cast<hipStream_t>(stream)));
}

int block_attn_fwd_workspace(int B, int H, int Hkv, int Sq, int Skv, int d, int n_list, size_t* bytes) {
  if (!bytes) return fail(TA_ERR_NULL_PTR, "bytes must be non-NULL");
  BlockGeo g;
  if (int st = make_geo(g, B, H, Hkv, Sq, Skv, d, n_list, 0, nullptr)) return st;
  *bytes = fwd_bytes(g);
  clear_error();
  return TA_OK;
}

int block_attn_fwd(const void* q, const void* k, const void* v, const int32_t* lists, void* out, float* lse, int B,
                   int H, int Hkv, int Sq, int Skv, int d, int n_list, int causal, const int32_t* lens, float scale,
                   void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !lists || !out) return fail(TA_ERR_NULL_PTR, "q, k, v, lists and out must be non-NULL");
  BlockFwdArgs a;
  if (int st = make_geo(a.g, B, H, Hkv, Sq, Skv, d, n_list, causal, lens)) return st;
  if (!std::isfinite(scale)) return fail(TA_ERR_BAD_SCALE, "scale must be finite");
  if (int st = check_aligned({q, k, v, out}, 16, "q, k, v and out must be 16-byte aligned")) return st;
  if (int st = check_aligned({lists, lse, lens}, 4, "lists, lse and lens must be 4-byte aligned")) return st;
  const size_t need = fwd_bytes(a.g);
  if (int st = check_workspace(workspace, workspace_bytes, need)) return st;
  const int64_t rows = (int64_t)B * H * Sq;
  const size_t qb = bf16s(rows * d), kb = bf16s((int64_t)B * Hkv * Skv * d);
  if (int st = check_apart({{out, qb}, {lse, (size_t)rows * 4}, {workspace, need}},
                           {{q, qb}, {k, kb}, {v, kb}, {lists, (size_t)lists_of(a.g) * n_list * 4}, {lens, (size_t)B * 4}}))
    return st;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.lists = lists;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  fold_scale(scale, a.c, a.qflip, a.qmask);
  a.units = units_of(a.g);
  a.pieces = pieces_of(a.g);
  a.part = static_cast<float*>(workspace);
  if (int st = check_grid((double)lists_of(a.g) * a.units * a.pieces)) return st;
  return launched(launch_block_fwd(a, static_cast<hipStream_t>(stream)));
}

int block_attn_bwd_workspace(int B, int H, int Hkv, int Sq, int Skv, int d, int n_list, size_t* bytes) {
  if (!bytes) return fail(TA_ERR_NULL_PTR, "bytes must be non-NULL");
  BlockGeo g;
  if (int st = make_geo(g, B, H, Hkv, Sq, Skv, d, n_list, 0, nullptr)) return st;
  *bytes = plan_bwd(g).bytes;
  clear_error();
  return TA_OK;
}

int block_attn_bwd(const void* q, const void* k, const void* v, const int32_t* lists, const void* out,
                   const void* dout, const float* lse, void* dq, void* dk, void* dv, int B, int H, int Hkv, int Sq,
                   int Skv, int d, int n_list, int causal, const int32_t* lens, float scale, void* workspace,
                   size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !lists || !out || !dout || !lse || !dq || !dk || !dv)
    return fail(TA_ERR_NULL_PTR, "q, k, v, lists, out, dout, lse, dq, dk and dv must be non-NULL");
  BlockBwdArgs a;
  if (int st = make_geo(a.g, B, H, Hkv, Sq, Skv, d, n_list, causal, lens)) return st;
  if (!std::isfinite(scale)) return fail(TA_ERR_BAD_SCALE, "scale must be finite");
  if (int st = check_aligned({q, k, v, out, dout, dq, dk, dv}, 16, "every bf16 tensor must be 16-byte aligned")) return st;
  if (int st = check_aligned({lists, lse, lens}, 4, "lists, lse and lens must be 4-byte aligned")) return st;
  const BwdPlan p = plan_bwd(a.g);
  if (int st = check_workspace(workspace, workspace_bytes, p.bytes)) return st;
  const int64_t rows = (int64_t)B * H * Sq, cols = (int64_t)B * Hkv * a.g.nb;
  const size_t qb = bf16s(rows * d), kb = bf16s((int64_t)B * Hkv * Skv * d);
  if (int st = check_apart({{dq, qb}, {dk, kb}, {dv, kb}, {workspace, p.bytes}},
                           {{q, qb},
                            {k, kb},
                            {v, kb},
                            {out, qb},
                            {dout, qb},
                            {lse, (size_t)rows * 4},
                            {lists, (size_t)lists_of(a.g) * n_list * 4},
                            {lens, (size_t)B * 4}}))
    return st;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.lists = lists;
  a.out = static_cast<const uint16_t*>(out);
  a.dout = static_cast<const uint16_t*>(dout);
  a.lse = lse;
  a.dq = static_cast<uint16_t*>(dq);
  a.dk = static_cast<uint16_t*>(dk);
  a.dv = static_cast<uint16_t*>(dv);
  fold_scale(scale, a.c, a.flip, a.keep);
  a.scale = scale;
  a.units = units_of(a.g);
  a.pieces_q = p.pieces_q;
  a.entries = p.entries;
  a.pieces_k = p.pieces_k;
  a.slots = (int)p.slots;
  // A column's start and end take about four units' time, and the masked tiles of its own query block
  // another block's.
  a.line = p.line;
  // Up to 32 KB of columns and 64 entries a thread.
  a.plan_in_prep = !p.line && cols * ((a.g.nq + 31) / 32) <= 8192 && lists_of(a.g) * n_list <= 16384;
  a.col_start = (16 + a.g.G - 1) / a.g.G + (causal ? 4 : 0);
  char* ws = static_cast<char*>(workspace);
  a.lse2 = reinterpret_cast<float*>(ws);
  a.ndelta = reinterpret_cast<float*>(ws + p.off_ndelta);
  a.cols = reinterpret_cast<uint32_t*>(ws + p.off_cols);
  a.plan = reinterpret_cast<int32_t*>(ws + p.off_plan);
  a.counts = reinterpret_cast<int32_t*>(ws + p.off_counts);
  a.items = reinterpret_cast<int32_t*>(ws + p.off_items);
  a.items_cap = (int)p.items_cap;
  a.part_q = reinterpret_cast<float*>(ws + p.off_q);
  a.part_k = reinterpret_cast<float*>(ws + p.off_k);
  if (int st = check_grid((double)lists_of(a.g) * a.units * a.pieces_q + 8.0 * p.items_cap)) return st;
  if (int st = check_grid(4.0 * lists_of(a.g) * a.units + 8.0 * cols)) return st;
  if (int st = check_grid((double)rows / 64 + (double)lists_of(a.g))) return st;
  return launched(launch_block_bwd(a, static_cast<hipStream_t>(stream)));
}

int cache_attn_write(const void* k, const void* v, void* k_pages, void* v_pages, float* k_scales, float* v_scales,
                     const int32_t* table, const int32_t* lens, const int32_t* n_new, int B, int Hkv, int N, int d,
                     int max_pages, int n_pages, void* stream) {
  if (!k || !v || !k_pages || !v_pages || !k_scales || !v_scales || !table || !lens)
    return fail(TA_ERR_NULL_PTR, "k, v, the pages, the scales, table and lens must be non-NULL");
  if (int st = check_cache(B, Hkv, Hkv, N, d, max_pages, kCacheSegment)) return st;
  if (n_pages < 1) return fail(TA_ERR_BAD_SHAPE, "n_pages must be >= 1");
  if (int st = check_aligned({k, v, k_pages, v_pages}, 16, "k, v and the pages must be 16-byte aligned")) return st;
  if (int st = check_aligned({k_scales, v_scales, table, lens, n_new}, 4,
                             "scales, table, lens and n_new must be 4-byte aligned"))
    return st;
  const size_t new_bytes = bf16s((int64_t)B * Hkv * N * d), pages = (size_t)n_pages * Hkv * TA_BLOCK * d;
  const size_t scales = (size_t)n_pages * Hkv * 4;
  if (int st = check_apart({{k_pages, pages}, {v_pages, pages}, {k_scales, scales}, {v_scales, scales}},
                           {{k, new_bytes},
                            {v, new_bytes},
                            {table, (size_t)B * max_pages * 4},
                            {lens, (size_t)B * 4},
                            {n_new, (size_t)B * 4}}))
    return st;
  const CacheWriteArgs a{static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v),
                         static_cast<uint8_t*>(k_pages), static_cast<uint8_t*>(v_pages), k_scales, v_scales, table,
                         lens, n_new, B, Hkv, N, d, max_pages, n_pages};
  return launched(launch_cache_write(a, static_cast<hipStream_t>(stream)));
}

int cache_attn_fwd_workspace(int B, int H, int Hkv, int N, int d, int max_pages, size_t* bytes) {
  if (!bytes) return fail(TA_ERR_NULL_PTR, "bytes must be non-NULL");
  if (int st = check_cache_attn(B, H, Hkv, N, d, max_pages, kCacheSegment)) return st;
  *bytes = plan_cache(B, H, Hkv, N, d, max_pages).bytes;
  clear_error();
  return TA_OK;
}

int cache_attn_fwd(const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
                   const float* v_scales, const int32_t* table, const int32_t* lens, int per_head, void* out,
                   float* lse, int B, int H, int Hkv, int N, int d, int max_pages, int n_pages, float scale,
                   void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k_pages || !v_pages || !k_scales || !v_scales || !table || !lens || !out)
    return fail(TA_ERR_NULL_PTR, "q, the pages, the scales, table, lens and out must be non-NULL");
  if (int st = check_cache_attn(B, H, Hkv, N, d, max_pages, kCacheSegment)) return st;
  if (n_pages < 1) return fail(TA_ERR_BAD_SHAPE, "n_pages must be >= 1");
  if (!std::isfinite(scale)) return fail(TA_ERR_BAD_SCALE, "scale must be finite");
  if (int st = check_aligned({q, k_pages, v_pages, out}, 16, "q, out and the pages must be 16-byte aligned")) return st;
  if (int st = check_aligned({k_scales, v_scales, table, lens, lse}, 4,
                             "scales, table, lens and lse must be 4-byte aligned"))
    return st;
  const CachePlan p = plan_cache(B, H, Hkv, N, d, max_pages);
  if (int st = check_workspace(workspace, workspace_bytes, p.bytes)) return st;
  const int64_t rows = (int64_t)B * H * N, entries = per_head ? (int64_t)B * Hkv : B;
  const size_t qb = bf16s(rows * d), pages = (size_t)n_pages * Hkv * TA_BLOCK * d, scales = (size_t)n_pages * Hkv * 4;
  if (int st = check_apart({{out, qb}, {lse, (size_t)rows * 4}, {workspace, p.bytes}},
                           {{q, qb},
                            {k_pages, pages},
                            {v_pages, pages},
                            {k_scales, scales},
                            {v_scales, scales},
                            {table, (size_t)entries * max_pages * 4},
                            {lens, (size_t)entries * 4}}))
    return st;
  CacheAttnArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.k_pages = static_cast<const uint8_t*>(k_pages);
  a.v_pages = static_cast<const uint8_t*>(v_pages);
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.table = table;
  a.lens = lens;
  a.per_head = per_head != 0;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.B = B;
  a.H = H;
  a.Hkv = Hkv;
  a.G = H / Hkv;
  a.N = N;
  a.d = d;
  a.max_pages = max_pages;
  a.n_pages = n_pages;
  a.c = scale * 1.4426950408889634f;
  a.whole = p.whole;
  a.workers = p.workers;
  a.row_blocks = p.passes;
  a.part = static_cast<float*>(workspace);
  return launched(launch_cache_attn(a, static_cast<hipStream_t>(stream)));
}

int cache4_attn_write(const void* k, const void* v, void* k_pages, void* v_pages, void* k_scales, void* v_scales,
                      const int32_t* table, const int32_t* lens, const int32_t* n_new, void* k_held, void* v_held,
                      int B, int Hkv, int N, int d, int max_pages, int n_pages, void* stream) {
  if (!k || !v || !k_pages || !v_pages || !k_scales || !v_scales || !table || !lens)
    return fail(TA_ERR_NULL_PTR, "k, v, the pages, the scales, table and lens must be non-NULL");
  if (int st = check_cache(B, Hkv, Hkv, N, d, max_pages, kCache4Segment)) return st;
  if (n_pages < 1) return fail(TA_ERR_BAD_SHAPE, "n_pages must be >= 1");
  if (int st = check_grid((double)N / cache4_tokens(d) + 1)) return st;
  if (int st = check_aligned({k, v, k_pages, v_pages, k_scales, v_scales, k_held, v_held}, 16,
                             "k, v, their held values, the pages and the scales must be 16-byte aligned"))
    return st;
  if (int st = check_aligned({table, lens, n_new}, 4, "table, lens and n_new must be 4-byte aligned")) return st;
  const size_t new_bytes = bf16s((int64_t)B * Hkv * N * d), pages = (size_t)n_pages * Hkv * TA_BLOCK * d / 2;
  const size_t scales = pages / (TA_CACHE4_GROUP / 2);
  if (int st = check_apart({{k_pages, pages}, {v_pages, pages}, {k_scales, scales}, {v_scales, scales},
                            {k_held, new_bytes}, {v_held, new_bytes}},
                           {{k, new_bytes},
                            {v, new_bytes},
                            {table, (size_t)B * max_pages * 4},
                            {lens, (size_t)B * 4},
                            {n_new, (size_t)B * 4}}))
    return st;
  const Cache4WriteArgs a{static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v),
                          static_cast<uint8_t*>(k_pages), static_cast<uint8_t*>(v_pages),
                          static_cast<uint8_t*>(k_scales), static_cast<uint8_t*>(v_scales), table, lens, n_new,
                          static_cast<uint16_t*>(k_held), static_cast<uint16_t*>(v_held), B, Hkv, N, d, max_pages,
                          n_pages, new_bytes * ((k_held != nullptr) + (v_held != nullptr)) > kStaysInCache};
  return launched(launch_cache4_write(a, static_cast<hipStream_t>(stream)));
}

int cache4_attn_read(const void* k_pages, const void* v_pages, const void* k_scales, const void* v_scales,
                     const int32_t* table, const int32_t* lens, void* k_out, void* v_out, int B, int Hkv, int N, int d,
                     int max_pages, int n_pages, int first, void* stream) {
  if (!k_pages || !v_pages || !k_scales || !v_scales || !table || !lens || (!k_out && !v_out))
    return fail(TA_ERR_NULL_PTR, "the pages, the scales, table, lens and k_out or v_out must be non-NULL");
  if (int st = check_cache(B, Hkv, Hkv, N, d, max_pages, kCache4Segment)) return st;
  if (n_pages < 1) return fail(TA_ERR_BAD_SHAPE, "n_pages must be >= 1");
  if (int st = check_grid((double)N / cache4_tokens(d) + 1)) return st;
  if (first < 0 || (int64_t)first + N > INT_MAX) return fail(TA_ERR_BAD_SHAPE, "first must be >= 0, first + N below 2^31");
  if (int st = check_aligned({k_pages, v_pages, k_scales, v_scales, k_out, v_out}, 16,
                             "the pages, the scales and the outputs must be 16-byte aligned"))
    return st;
  if (int st = check_aligned({table, lens}, 4, "table and lens must be 4-byte aligned")) return st;
  const size_t out = bf16s((int64_t)B * Hkv * N * d), pages = (size_t)n_pages * Hkv * TA_BLOCK * d / 2;
  const size_t scales = pages / (TA_CACHE4_GROUP / 2);
  if (int st = check_apart({{k_out, out}, {v_out, out}},
                           {{k_pages, pages},
                            {v_pages, pages},
                            {k_scales, scales},
                            {v_scales, scales},
                            {table, (size_t)B * max_pages * 4},
                            {lens, (size_t)B * 4}}))
    return st;
  const Cache4ReadArgs a{static_cast<const uint8_t*>(k_pages), static_cast<const uint8_t*>(v_pages),
                         static_cast<const uint8_t*>(k_scales), static_cast<const uint8_t*>(v_scales), table, lens,
                         static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out), B, Hkv, N, d, max_pages,
                         n_pages, first, out * ((k_out != nullptr) + (v_out != nullptr)) > kStaysInCache};
  return launched(launch_cache4_read(a, static_cast<hipStream_t>(stream)));
}

int cache4_attn_fwd_workspace(int B, int H, int Hkv, int N, int d, int max_pages, size_t* bytes) {
  if (!bytes) return fail(TA_ERR_NULL_PTR, "bytes must be non-NULL");
  if (int st = check_cache_attn(B, H, Hkv, N, d, max_pages, kCache4Segment)) return st;
  *bytes = plan_cache4(B, H, Hkv, N, d, max_pages).bytes;
  clear_error();
  return TA_OK;
}

int cache4_attn_fwd(const void* q, const void* k_pages, const void* v_pages, const void* k_scales,
                    const void* v_scales, const int32_t* table, const int32_t* lens, int per_head, void* out,
                    float* lse, int B, int H, int Hkv, int N, int d, int max_pages, int n_pages, float scale,
                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k_pages || !v_pages || !k_scales || !v_scales || !table || !lens || !out)
    return fail(TA_ERR_NULL_PTR, "q, the pages, the scales, table, lens and out must be non-NULL");
  if (int st = check_cache_attn(B, H, Hkv, N, d, max_pages, kCache4Segment)) return st;
  if (n_pages < 1) return fail(TA_ERR_BAD_SHAPE, "n_pages must be >= 1");
  if (!std::isfinite(scale)) return fail(TA_ERR_BAD_SCALE, "scale must be finite");
  if (int st = check_aligned({q, k_pages, v_pages, k_scales, v_scales, out}, 16,
                             "q, out, the pages and the scales must be 16-byte aligned"))
    return st;
  if (int st = check_aligned({table, lens, lse}, 4, "table, lens and lse must be 4-byte aligned")) return st;
  const CachePlan p = plan_cache4(B, H, Hkv, N, d, max_pages);
  if (int st = check_workspace(workspace, workspace_bytes, p.bytes)) return st;
  const int64_t rows = (int64_t)B * H * N, entries = per_head ? (int64_t)B * Hkv : B;
  const size_t qb = bf16s(rows * d), pages = (size_t)n_pages * Hkv * TA_BLOCK * d / 2;
  const size_t scales = pages / (TA_CACHE4_GROUP / 2);
  if (int st = check_apart({{out, qb}, {lse, (size_t)rows * 4}, {workspace, p.bytes}},
                           {{q, qb},
                            {k_pages, pages},
                            {v_pages, pages},
                            {k_scales, scales},
                            {v_scales, scales},
                            {table, (size_t)entries * max_pages * 4},
                            {lens, (size_t)entries * 4}}))
    return st;
  Cache4AttnArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.k_pages = static_cast<const uint8_t*>(k_pages);
  a.v_pages = static_cast<const uint8_t*>(v_pages);
  a.k_scales = a.v_scales = nullptr;
  a.k_exps = static_cast<const uint8_t*>(k_scales);
  a.v_exps = static_cast<const uint8_t*>(v_scales);
  a.table = table;
  a.lens = lens;
  a.per_head = per_head != 0;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.B = B;
  a.H = H;
  a.Hkv = Hkv;
  a.G = H / Hkv;
  a.N = N;
  a.d = d;
  a.max_pages = max_pages;
  a.n_pages = n_pages;
  fold_scale(scale, a.c, a.q_flip, a.q_keep);
  a.whole = p.whole;
  a.eight = p.eight;
  a.workers = p.workers;
  a.row_blocks = p.passes;
  a.part = static_cast<float*>(workspace);
  return launched(launch_cache4_attn(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
