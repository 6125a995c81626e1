// Host side of the C ABI of attention over selected blocks and over the 8-bit cache: argument
// checks, how work is cut, and the workspaces' sizes. Nothing is allocated and nothing is kept.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <initializer_list>
#include <string>

#include "block_attn.h"
#include "block_launch.h"
#include "host_internal.h"

namespace ta {
namespace host {
namespace {

static_assert(kBlock == TA_BLOCK, "block size");
static_assert(kBlockWords * 32 == TA_MAX_BLOCKS, "bitmap size");

// Workgroups that the device runs at a time at two per compute unit (256 units). Work is cut by
// this number, not by the device's own, so that workspaces have the same size everywhere.
constexpr int64_t kSlots = 512;
constexpr int64_t kMaxGrid = (int64_t)UINT32_MAX / 256 - 8;

struct Span {
  const void* p;
  size_t bytes;
};
size_t bf16s(int64_t n) { return (size_t)n * 2; }

int check_aligned(std::initializer_list<const void*> ps, unsigned align, const char* what) {
  for (const void* p : ps)
    if (p && reinterpret_cast<uintptr_t>(p) % align) return fail(TA_ERR_ALIGN, what);
  return TA_OK;
}
// Outputs (and the workspace) must overlap neither an input nor each other.
int check_apart(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    if (!o->p || !o->bytes) continue;
    for (const Span& x : ins)
      if (x.p && x.bytes && ranges_overlap(o->p, o->bytes, x.p, x.bytes))
        return fail(TA_ERR_OVERLAP, "an output or the workspace overlaps an input");
    for (auto q = o + 1; q != outs.end(); ++q)
      if (q->p && q->bytes && ranges_overlap(o->p, o->bytes, q->p, q->bytes))
        return fail(TA_ERR_OVERLAP, "outputs and the workspace must not overlap each other");
  }
  return TA_OK;
}
int launched(hipError_t e) {
  if (e != hipSuccess) return fail(TA_ERR_HIP, std::string("kernel launch: ") + hipGetErrorString(e));
  clear_error();
  return TA_OK;
}

int check_grid(double workgroups) {
  return workgroups <= (double)kMaxGrid ? TA_OK : fail(TA_ERR_BAD_SHAPE, "the call exceeds the grid limit");
}
int check_dim(int d) {
  return d == 64 || d == 96 || d == 128 ? TA_OK : fail(TA_ERR_HEAD_DIM, "d must be 64, 96 or 128");
}

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

int check_workspace(const void* ws, size_t have, size_t need) {
  if (have < need || (need && !ws))
    return fail(TA_ERR_BAD_SHAPE, "the workspace is smaller than the call needs (" + std::to_string(need) + " bytes)");
  return check_aligned({ws}, 16, "the workspace must be 16-byte aligned");
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
  bool whole;
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
  if (p.whole) p.workers = B * Hkv;
  p.bytes = p.whole || p.workers == 1 ? 0 : (size_t)p.passes * 2 * p.workers * p.rows * (d + 4) * sizeof(float);
  return p;
}
int check_cache(int B, int H, int Hkv, int N, int d, int max_pages) {
  if (B < 1 || H < 1 || Hkv < 1 || N < 1 || max_pages < 1)
    return fail(TA_ERR_BAD_SHAPE, "B, H, Hkv, N and max_pages must be >= 1");
  if (H % Hkv) return fail(TA_ERR_BAD_SHAPE, "H must be a multiple of Hkv");
  if (max_pages > INT_MAX / TA_BLOCK) return fail(TA_ERR_BAD_SHAPE, "max_pages pages hold more than 2^31 - 1 tokens");
  // The sequences times heads are a grid dimension of their own.
  if ((int64_t)B * Hkv * (max_pages + kCacheSegment) > INT_MAX)
    return fail(TA_ERR_BAD_SHAPE, "B * Hkv * max_pages exceeds 2^31 - 1");
  if ((int64_t)B * Hkv > 65535) return fail(TA_ERR_BAD_SHAPE, "B * Hkv exceeds the grid limit");
  return check_dim(d);
}
// Attention: so are the passes over its rows and the joins of 8 of them.
int check_cache_attn(int B, int H, int Hkv, int N, int d, int max_pages) {
  if (int st = check_cache(B, H, Hkv, N, d, max_pages)) return st;
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
  if (int st = check_cache(B, Hkv, Hkv, N, d, max_pages)) return st;
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
  if (int st = check_cache_attn(B, H, Hkv, N, d, max_pages)) return st;
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
  if (int st = check_cache_attn(B, H, Hkv, N, d, max_pages)) return st;
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

}  // extern "C"
