// Host side of the C ABI of head norms and rotations: argument checks and how work is cut. Nothing is allocated
// and nothing is kept.
#include <algorithm>
#include <array>
#include <cfloat>
#include <cmath>
#include <string>

#include "head_rope.h"
#include "host_checks.h"
#include "host_internal.h"
#include "rope_launch.h"

namespace ta {
namespace host {
namespace {

static_assert(kRopeAxes == TA_ROPE_AXES, "axes");

// Everything that spec says, checked, but for the tensors.
int from_spec(const head_rope_spec* spec, RopeArgs& a) {
  if (!spec) return fail(TA_ERR_NULL_PTR, "spec must be non-NULL");
  const head_rope_spec& s = *spec;
  if (s.B < 1 || s.S < 1 || s.H < 1 || s.Hkv < 1) return fail(TA_ERR_BAD_SHAPE, "B, S, H and Hkv must be >= 1");
  if (int st = check_dim(s.d)) return st;
  if ((int64_t)s.B * s.S > INT32_MAX || (int64_t)s.S * s.d > INT32_MAX)
    return fail(TA_ERR_BAD_SHAPE, "B * S and S * d must stay below 2^31");
  if ((int64_t)s.H + 2 * (int64_t)s.Hkv > 65535) return fail(TA_ERR_BAD_SHAPE, "H + 2 * Hkv exceeds the grid limit");
  if (s.norm < TA_NORM_NONE || s.norm > TA_NORM_LAYER) return fail(TA_ERR_BAD_SHAPE, "norm is none of ta_norm");
  if (s.layout < TA_ROPE_NONE || s.layout > TA_ROPE_SPLIT) return fail(TA_ERR_BAD_SHAPE, "layout is none of ta_rope_layout");
  if (s.norm == TA_NORM_NONE && (s.q_weight || s.k_weight)) return fail(TA_ERR_BAD_SHAPE, "weights need a norm");
  if (s.norm != TA_NORM_LAYER && (s.q_bias || s.k_bias)) return fail(TA_ERR_BAD_SHAPE, "biases need TA_NORM_LAYER");
  if (s.norm != TA_NORM_NONE && !(s.eps >= FLT_MIN && s.eps <= FLT_MAX))
    return fail(TA_ERR_BAD_SCALE, "eps must be a finite number, not below the smallest normal one");
  a.B = s.B;
  a.S = s.S;
  a.d = s.d;
  a.norm = s.norm;
  a.layout = s.layout;
  a.axes = 0;
  a.turned = 0;
  a.whole = true;
  a.freqs = nullptr;
  a.positions = nullptr;
  a.positions_batch = 0;
  for (int x = 0; x < kRopeAxes; ++x) {
    a.dims[x] = 0;
    a.start[x] = INT32_MAX;  // behind every value
  }
  if (s.layout != TA_ROPE_NONE) {
    if (s.axes < 1 || s.axes > TA_ROPE_AXES) return fail(TA_ERR_BAD_SHAPE, "axes must be in 1..TA_ROPE_AXES");
    a.axes = s.axes;
    for (int x = 0; x < s.axes; ++x) {
      if (s.dims[x] < 2 || s.dims[x] > s.d || s.dims[x] % 2)
        return fail(TA_ERR_BAD_SHAPE, "dims must be even and in 2..d");
      a.dims[x] = s.dims[x];
      a.start[x] = a.turned;
      a.turned += s.dims[x];
      // Halves that are multiples of 8 start at multiples of 16. Where all turned values have one half it takes all
      // of them too: eight values belong to one axis only if each has a multiple of 8 pairs.
      if (s.dims[x] % 16) a.whole = false;
    }
    if (a.turned > s.d) return fail(TA_ERR_BAD_SHAPE, "the axes' dims must add up to d at most");
    if (!s.freqs || !s.positions) return fail(TA_ERR_NULL_PTR, "freqs and positions must be non-NULL");
    if (s.positions_batch < 0) return fail(TA_ERR_BAD_SHAPE, "positions_batch must not be negative");
    if (int st = check_aligned({s.freqs}, 8, "freqs must be 8-byte aligned")) return st;
    if (int st = check_aligned({s.positions}, 4, "positions must be 4-byte aligned")) return st;
    a.freqs = s.freqs;
    a.positions = s.positions;
    a.positions_batch = s.positions_batch;
  }
  if (int st = check_aligned({s.q_weight, s.k_weight, s.q_bias, s.k_bias}, 16, "weights and biases must be 16-byte aligned"))
    return st;
  if (int st = check_aligned({s.lens}, 4, "lens must be 4-byte aligned")) return st;
  a.eps = s.eps;
  a.weight[0] = s.q_weight;
  a.weight[1] = s.k_weight;
  a.bias[0] = s.q_bias;
  a.bias[1] = s.k_bias;
  a.lens = s.lens;
  a.heads[0] = s.H;
  a.heads[1] = a.heads[2] = s.Hkv;
  for (int x = 0; x < 3; ++x) {
    a.x[x] = a.dx[x] = Rows{nullptr, 0, 0, 0};
    a.y[x] = nullptr;
  }
  a.heads_per = 1;
  for (int& x : a.first) x = 0;
  a.part = nullptr;
  for (float*& x : a.sum) x = nullptr;
  return TA_OK;
}

// Values between the first and the last of rows' tensor, both in it; 0 if that passes 2^62.
int64_t extent(const RopeArgs& a, const ta_rows& r, int heads) {
  const double most = (double)(a.B - 1) * (double)r.batch + (double)(a.S - 1) * (double)r.token +
                      (double)(heads - 1) * (double)r.head + a.d;
  if (most > 4.6e18) return 0;
  return (a.B - 1) * r.batch + (a.S - 1) * r.token + (heads - 1) * r.head + a.d;
}

int check_rows(const RopeArgs& a, const ta_rows& r, int heads, const char* what, Span& span) {
  if (!r.data) return fail(TA_ERR_NULL_PTR, std::string(what) + " must be non-NULL");
  if (int st = check_aligned({r.data}, 16, "rows must be 16-byte aligned")) return st;
  if (r.batch < 0 || r.token < 0 || r.head < 0 || r.batch % 8 || r.token % 8 || r.head % 8)
    return fail(TA_ERR_ALIGN, "strides must be multiples of 8 values, not negative");
  const int64_t n = extent(a, r, heads);
  if (n == 0) return fail(TA_ERR_BAD_SHAPE, "strides reach past the address space");
  span = Span{r.data, bf16s(n)};
  return TA_OK;
}

// Whether places at these steps (of n each) hold pieces of `inside` values apart: in order of the steps, each is at
// least as long as all that lies inside it.
struct Axis {
  int64_t step;
  int n;
};
bool pieces_apart(std::array<Axis, 3> axes, int64_t inside) {
  std::sort(axes.begin(), axes.end(), [](const Axis& x, const Axis& y) { return x.step < y.step; });
  for (const Axis& x : axes) {
    if (x.n == 1) continue;
    if (x.step < inside) return false;
    inside += (x.n - 1) * x.step;
  }
  return true;
}
// No value of written rows stands for two rows.
bool one_place_each(const RopeArgs& a, const ta_rows& r, int heads) {
  return pieces_apart({{{r.batch, a.B}, {r.token, a.S}, {r.head, heads}}}, a.d);
}

// Whether two written tensors share no value: their extents are apart, or they stand in one tensor, heads behind
// heads of the same tokens.
bool apart(const RopeArgs& a, const ta_rows& p, int np, const ta_rows& q, int nq) {
  if (!ranges_overlap(p.data, bf16s(extent(a, p, np)), q.data, bf16s(extent(a, q, nq)))) return true;
  const bool first = reinterpret_cast<uintptr_t>(p.data) <= reinterpret_cast<uintptr_t>(q.data);
  const ta_rows& lo = first ? p : q;
  const ta_rows& hi = first ? q : p;
  const int64_t off = (int64_t)(reinterpret_cast<uintptr_t>(hi.data) - reinterpret_cast<uintptr_t>(lo.data)) / 2;
  if ((a.B > 1 && lo.batch != hi.batch) || (a.S > 1 && lo.token != hi.token)) return false;
  // A token's heads of lo, then those of hi, are one piece, and pieces do not meet.
  const int64_t lo_piece = ((first ? np : nq) - 1) * lo.head + a.d, hi_piece = ((first ? nq : np) - 1) * hi.head + a.d;
  return off >= lo_piece && pieces_apart({{{lo.batch, a.B}, {lo.token, a.S}, {0, 1}}}, off + hi_piece);
}

Rows to_rows(const ta_rows& r) {
  return Rows{static_cast<uint16_t*>(const_cast<void*>(r.data)), r.batch, r.token, r.head};
}

// Bytes of what spec points to, as inputs.
struct SpecSpans {
  Span at[7];
  explicit SpecSpans(const head_rope_spec& s, const RopeArgs& a) {
    const size_t w = (size_t)s.d * 4;
    at[0] = Span{s.q_weight, w};
    at[1] = Span{s.k_weight, w};
    at[2] = Span{s.q_bias, w};
    at[3] = Span{s.k_bias, w};
    at[4] = Span{a.freqs, (size_t)a.turned / 2 * 8};
    at[5] = Span{a.positions, ((size_t)(s.B - 1) * (size_t)a.positions_batch + (size_t)s.S * a.axes) * 4};
    at[6] = Span{s.lens, (size_t)s.B * 4};
  }
};

int64_t groups_of(const RopeArgs& a) {
  const int tokens = rope_tokens(a.d);
  return ((int64_t)a.B * a.S + tokens - 1) / tokens;
}

// Heads that a wave takes of its tokens: few, so that kFewWaves waves form (and two at least: one after the other
// they wait for less); past that a wave's start, its angles and weights, should be worth `worth` heads, up to kManyWaves.
// 2 sequences of 777, 10 heads, d = 64: 4.8 us with two heads a wave, 6.3 with four, 7.5 with eight. 4000 tokens, 72 heads, d = 96,
// pairs anywhere in the row: 23.6 with 18 heads a wave, 24.9 with 36; 17776 tokens, 144 heads, d = 64, neighbours: 150 us with 144, 136
// with 48, 132 with 21.
constexpr int64_t kFewWaves = 2048, kManyWaves = 16 * 1024;
int heads_per_wave(const RopeArgs& a, int heads) {
  const int64_t groups = groups_of(a);
  auto of = [&](int64_t waves) {
    const int64_t parts = std::max<int64_t>(1, (waves + groups - 1) / groups);
    return (heads + parts - 1) / parts;
  };
  const bool near = a.layout == TA_ROPE_NONE || a.layout == TA_ROPE_INTERLEAVED;
  const int64_t worth = near ? 12 : 18;
  return (int)std::max<int64_t>({std::min(heads, 2), of(kManyWaves), std::min(of(kFewWaves), worth)});
}

// Gradients: the heads that a wave takes at a time, and workgroups, four a compute unit at most, as many as are
// resident at once, shared out by the bytes of a row of q, k (read twice, written) and v (read, written). 28800 tokens, 72
// heads, d = 96: 233 us so; 286 with 768 workgroups, 294 with 1280, 239 with 2048; 240 with 4 heads a wave, 234 with 24; shares by heads
// alone 240. 512 tokens, 48 heads of 128: 13.9 us with 3 heads a wave, 17.5 with one.
constexpr int64_t kGradWorkgroups = 1024;
void plan_grad(RopeArgs& a) {
  const int64_t groups = groups_of(a), heads = (int64_t)a.heads[0] + a.heads[1] + a.heads[2];
  a.heads_per = (int)std::max<int64_t>(1, std::min<int64_t>(8, 2 * groups * heads / (kGradWorkgroups * kRopeWaves)));
  int64_t need[3], share[3], total = 0;
  for (int x = 0; x < 3; ++x) {
    need[x] = (groups * ((a.heads[x] + a.heads_per - 1) / a.heads_per) + kRopeWaves - 1) / kRopeWaves;
    share[x] = (int64_t)(x < 2 && a.norm != TA_NORM_NONE ? 3 : 2) * a.heads[x];
    total += share[x];
  }
  a.first[0] = 0;
  for (int x = 0; x < 3; ++x) {
    const int64_t n = a.heads[x] ? std::max<int64_t>(1, kGradWorkgroups * share[x] / total) : 0;
    a.first[x + 1] = a.first[x] + (int)std::min(n, need[x]);
  }
}
// A row of partial sums for each workgroup of q's and k's rows: whatever of q, k and v is left out, at most
// this many (a share is rounded down, but not to none), and no more than items of one head make.
size_t grad_bytes(const RopeArgs& a, int H, int Hkv) {
  if (a.norm == TA_NORM_NONE) return 0;
  auto most = [&](int heads) { return (groups_of(a) * heads + kRopeWaves - 1) / kRopeWaves; };
  return (size_t)std::min(kGradWorkgroups + 2, most(H) + most(Hkv)) * 2 * a.d * sizeof(float);
}

}  // namespace
}  // namespace host
}  // namespace ta

using namespace ta;
using namespace ta::host;

extern "C" {

int head_rope_fwd(const head_rope_spec* spec, const ta_rows* q, const ta_rows* k, const ta_rows* v, void* q_out,
                  void* k_out, void* v_out, void* stream) {
  RopeArgs a;
  if (int st = from_spec(spec, a)) return st;
  const ta_rows* in[3] = {q, k, v};
  void* out[3] = {q_out, k_out, v_out};
  const char* names[3] = {"q", "k", "v"};
  Span ins[3] = {}, outs[3] = {};
  int heads = 0;
  for (int x = 0; x < 3; ++x) {
    if (!in[x] != !out[x]) return fail(TA_ERR_NULL_PTR, std::string(names[x]) + " and its output go together");
    if (!in[x]) {
      a.heads[x] = 0;
      continue;
    }
    if (int st = check_rows(a, *in[x], a.heads[x], names[x], ins[x])) return st;
    if (int st = check_aligned({out[x]}, 16, "outputs must be 16-byte aligned")) return st;
    a.x[x] = to_rows(*in[x]);
    a.y[x] = static_cast<uint16_t*>(out[x]);
    outs[x] = Span{out[x], bf16s((int64_t)a.B * a.heads[x] * a.S * a.d)};
    heads += a.heads[x];
  }
  if (heads == 0) return fail(TA_ERR_NULL_PTR, "one of q, k and v must be there");
  const SpecSpans given(*spec, a);
  if (int st = check_apart({outs[0], outs[1], outs[2]},
                           {ins[0], ins[1], ins[2], given.at[0], given.at[1], given.at[2], given.at[3], given.at[4],
                            given.at[5], given.at[6]}))
    return st;
  a.heads_per = heads_per_wave(a, heads);
  if (int st = check_grid((double)groups_of(a) / kRopeWaves + 1)) return st;
  return launched(launch_head_rope(a, static_cast<hipStream_t>(stream)));
}

int head_rope_bwd_workspace(const head_rope_spec* spec, size_t* bytes) {
  if (!bytes) return fail(TA_ERR_NULL_PTR, "bytes must be non-NULL");
  RopeArgs a;
  if (int st = from_spec(spec, a)) return st;
  *bytes = grad_bytes(a, a.heads[0], a.heads[1]);
  clear_error();
  return TA_OK;
}

int head_rope_bwd(const head_rope_spec* spec, const ta_rows* q, const ta_rows* k, const void* dq_out,
                  const void* dk_out, const void* dv_out, const ta_rows* dq, const ta_rows* dk, const ta_rows* dv,
                  float* dq_weight, float* dk_weight, float* dq_bias, float* dk_bias, void* workspace,
                  size_t workspace_bytes, void* stream) {
  RopeArgs a;
  if (int st = from_spec(spec, a)) return st;
  const size_t need = grad_bytes(a, a.heads[0], a.heads[1]);
  const ta_rows* in[3] = {q, k, nullptr};
  const void* g[3] = {dq_out, dk_out, dv_out};
  const ta_rows* out[3] = {dq, dk, dv};
  float* sums[4] = {dq_weight, dq_bias, dk_weight, dk_bias};
  const char* names[3] = {"dq", "dk", "dv"};
  Span ins[3] = {}, gs[3] = {}, outs[3] = {}, adds[4] = {};
  for (int x = 0; x < 3; ++x) {
    if (!g[x] != !out[x]) return fail(TA_ERR_NULL_PTR, std::string(names[x]) + " and the result's gradient go together");
    if (!g[x]) {
      a.heads[x] = 0;
      continue;
    }
    if (x < 2 && a.norm != TA_NORM_NONE) {
      if (!in[x]) return fail(TA_ERR_NULL_PTR, "with a norm q and k must be there");
      if (int st = check_rows(a, *in[x], a.heads[x], x == 0 ? "q" : "k", ins[x])) return st;
      a.x[x] = to_rows(*in[x]);
    }
    if (int st = check_aligned({g[x]}, 16, "gradients must be 16-byte aligned")) return st;
    if (int st = check_rows(a, *out[x], a.heads[x], names[x], outs[x])) return st;
    if (!one_place_each(a, *out[x], a.heads[x])) return fail(TA_ERR_OVERLAP, "rows that are written overlap each other");
    a.y[x] = static_cast<uint16_t*>(const_cast<void*>(g[x]));
    a.dx[x] = to_rows(*out[x]);
    gs[x] = Span{g[x], bf16s((int64_t)a.B * a.heads[x] * a.S * a.d)};
  }
  if (a.heads[0] + a.heads[1] + a.heads[2] == 0) return fail(TA_ERR_NULL_PTR, "one of q, k and v must be there");
  bool wanted = false;
  for (int x = 0; x < 4; ++x) {
    if (!sums[x]) continue;
    if (a.norm == TA_NORM_NONE || (x % 2 && a.norm != TA_NORM_LAYER) || a.heads[x / 2] == 0)
      return fail(TA_ERR_BAD_SHAPE, "weights' gradients need a norm, biases' TA_NORM_LAYER, and both their rows");
    if (int st = check_aligned({sums[x]}, 16, "gradients of weights and biases must be 16-byte aligned")) return st;
    adds[x] = Span{sums[x], (size_t)a.d * 4};
    a.sum[x] = sums[x];
    wanted = true;
  }
  if (int st = check_workspace(workspace, workspace_bytes, need)) return st;
  plan_grad(a);
  a.part = wanted ? static_cast<float*>(workspace) : nullptr;
  for (int x = 0; x < 3; ++x)
    for (int y = x + 1; y < 3; ++y)
      if (out[x] && out[y] && !apart(a, *out[x], a.heads[x], *out[y], a.heads[y]))
        return fail(TA_ERR_OVERLAP, "dq, dk and dv overlap each other");
  const SpecSpans given(*spec, a);
  const Span ws{workspace, need};
  for (int x = 0; x < 3; ++x)
    if (int st = check_apart({outs[x], adds[0], adds[1], adds[2], adds[3], ws},
                             {ins[0], ins[1], gs[0], gs[1], gs[2], given.at[0], given.at[1], given.at[2], given.at[3],
                              given.at[4], given.at[5], given.at[6]}))
      return st;
  return launched(launch_head_rope_grad(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
