// gfx950 (MI355X, CDNA4) kernels of head norms and rotations, forward and gradients.
//
// A row (the d values of a head of a token) takes 8 lanes at d = 64 and 16 at 96 (12 of them at work) and
// 128, 8 values a lane: 16-byte loads and stores, and sums over a row in four or three steps inside the lanes of
// a DPP row. A wave holds rows of 4 (8) tokens that follow each other, of one head at a time, and goes through the
// heads: what depends on the token alone, cosines and sines of its angles times the weights, is formed once for
// all of them, and stores of one head are whole stretches of its [S, d] plane. No sum crosses a DPP row, so nothing
// but a pair's other value goes through LDS, and that only where it is in another lane.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "rope_launch.h"
#include "tile_common.h"

namespace ta {
namespace {

constexpr int kNone = 0, kRms = 1, kLayer = 2;  // norms
// How a value's partner is found: no rotation; its neighbour; 8 values that another lane holds; anywhere in
// the row.
constexpr int kStill = 0, kNext = 1, kWhole = 2, kAny = 3;

typedef float Floats8[8];
constexpr double kTurn = 0.15915494309189533577;  // 1 / 2 pi

template <int D>
struct Shape {
  static constexpr int lanes = D == 64 ? 8 : 16;  // of a row
  static constexpr int tokens = 64 / lanes;
  static_assert(tokens == rope_tokens(D), "tokens of a wave");
  // A row in LDS: its 16-byte pieces and one of zeros (d = 96: lanes behind the row write it).
  static constexpr int none = D / 8, pitch = D == 96 ? lanes : none + 1, pieces = tokens * pitch;
};

// The sum over a row's lanes, in all of them: neighbours, pairs, then mirrored halves (of 8 and of 16 lanes).
template <int CTRL>
__device__ __forceinline__ float add_from(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int D>
__device__ __forceinline__ float row_sum(float x) {
  x = add_from<0xb1>(x);   // lanes 1 0 3 2 of each four
  x = add_from<0x4e>(x);   // lanes 2 3 0 1
  x = add_from<0x141>(x);  // mirrored in 8 lanes
  if constexpr (D != 64) x = add_from<0x140>(x);  // mirrored in 16 lanes
  return x;
}

__device__ __forceinline__ void widen(u32x4 w, Floats8& x) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
// One rounding to bf16, to nearest, ties to even.
__device__ __forceinline__ u32x4 narrow(const Floats8& x) {
  const f32x8 y = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
  return __builtin_bit_cast(u32x4, __builtin_convertvector(y, bf16x8));
}

// What value e of a head is in the rotation: its partner, its pair and the pair's axis, whether it is turned at all
// and the pair's second value. Without branches (unused axes start behind every value): a lane asks for up to 8
// values, and what it then loads should not wait for one another.
struct Place {
  int partner, pair, axis;
  bool turned, second;
};
__device__ __forceinline__ Place place_of(const RopeArgs& a, int e) {
  const bool split = a.layout == 3, interleaved = a.layout == 1;
  const int h = a.turned / 2;
  const int at = split ? 2 * (e >= h ? e - h : e) : e;  // decides the axis
  int axis = 0, start = 0, n = a.dims[0];
#pragma unroll
  for (int x = 1; x < kRopeAxes; ++x) {
    const bool past = at >= a.start[x];
    axis = past ? x : axis;
    start = past ? a.start[x] : start;
    n = past ? a.dims[x] : n;
  }
  const int half = split ? h : n / 2, o = split ? e : e - start;
  Place p;
  p.second = interleaved ? (e & 1) != 0 : o >= half;
  p.partner = interleaved ? e ^ 1 : p.second ? e - half : e + half;  // (axes start at even values)
  p.pair = interleaved ? e / 2 : (split ? 0 : start / 2) + (p.second ? o - half : o);
  p.axis = axis;
  p.turned = e < a.turned;
  if (!p.turned) {
    p.partner = e;
    p.pair = 0;
  }
  return p;
}

// A value's place where pairs are anywhere in the row: formed once a workgroup, by a thread a value, and kept in LDS.
struct __attribute__((aligned(16))) PlaceEntry {
  double f;         // turns per position
  uint16_t from;    // byte of the partner in its row, of the zeros for a value that is not turned
  uint16_t axis;
  float sign;       // of the partner's sine
};

// The lane's 8 values in the rotation. Angles: turns = position * (frequency / 2 pi) in fp64, three roundings (1 / 2 pi's, two
// products') of at most 2^-53 of the angle however far the position, then the fraction alone, in fp32, for v_sin_f32 and v_cos_f32
// (which take turns; off by at most 1.3e-7 in [-0.5, 0.5]: nothing beside a result's rounding to bf16).
template <int D, int ROT>
struct Turns {
  static constexpr int kAngles = ROT == kNext ? 4 : 8;
  double f[ROT == kStill ? 1 : kAngles];
  int axis[ROT == kStill ? 1 : ROT == kWhole ? 1 : kAngles];
  int from[ROT == kAny ? 8 : 1];  // byte of the partner in its row, or the piece with all eight
  float sign[ROT == kAny ? 8 : 1];
  bool every;  // kNext: all values of a head are turned
  int left;    // kNext: how many of the lane's are

  // (With kAny all threads of a workgroup call it together.)
  __device__ __forceinline__ void place(const RopeArgs& a, int l, PlaceEntry* entries) {
    if constexpr (ROT == kAny) {
      if (threadIdx.x < D) {
        const Place p = place_of(a, threadIdx.x);
        const double x = a.freqs[p.pair];
        entries[threadIdx.x] = PlaceEntry{p.turned ? x * kTurn : 0., (uint16_t)(p.turned ? 2 * p.partner : 16 * Shape<D>::none),
                                          (uint16_t)p.axis, p.second ? 1.f : -1.f};
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const PlaceEntry p = entries[min(8 * l + i, D - 1)];
        f[i] = p.f;
        axis[i] = p.axis;
        from[i] = p.from;
        sign[i] = 8 * l >= D ? 0.f : p.sign;
      }
    } else if constexpr (ROT == kWhole) {
      // Eight values of one axis and half, their pairs one after the other. (A lane behind the row takes
      // nothing from it: sums over the row's lanes add it too.)
      const Place p = place_of(a, min(8 * l, D - 8));
      from[0] = p.turned ? p.partner / 8 : Shape<D>::none;
      axis[0] = p.axis;
      sign[0] = 8 * l >= D ? 0.f : p.second ? 1.f : -1.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double x = a.freqs[p.turned ? p.pair + i : 0];
        f[i] = p.turned ? x * kTurn : 0.;
      }
    } else if constexpr (ROT == kNext) {
      every = a.turned >= D;
      left = a.turned - 8 * l;
      Place p[kAngles];
#pragma unroll
      for (int i = 0; i < kAngles; ++i) p[i] = place_of(a, min(8 * l + 2 * i, D - 1));
#pragma unroll
      for (int i = 0; i < kAngles; ++i) {
        const double x = a.freqs[p[i].pair];
        f[i] = p[i].turned ? x * kTurn : 0.;
        axis[i] = p[i].axis;
      }
    }
  }
  // c, s: y_e = n_e c_e + n_partner s_e.
  __device__ __forceinline__ void at(const RopeArgs& a, int b, int t, Floats8& c, Floats8& s) const {
    if constexpr (ROT != kStill) {
      const int32_t* p = a.positions + b * a.positions_batch + (int64_t)t * a.axes;
      int pos[kRopeAxes];
#pragma unroll
      for (int x = 0; x < kRopeAxes; ++x) pos[x] = p[min(x, a.axes - 1)];
#pragma unroll
      for (int i = 0; i < kAngles; ++i) {
        const int of = axis[ROT == kWhole ? 0 : i];
        int at = pos[0];
#pragma unroll
        for (int x = 1; x < kRopeAxes; ++x) at = of == x ? pos[x] : at;
        const double turns = (double)at * f[i];
        const float part = (float)(turns - __builtin_rint(turns));
        const float cs = __builtin_amdgcn_cosf(part), sn = __builtin_amdgcn_sinf(part);
        if constexpr (ROT == kNext) {
          c[2 * i] = c[2 * i + 1] = cs;
          s[2 * i] = -sn;
          s[2 * i + 1] = sn;
        } else {
          c[i] = cs;
          s[i] = sign[ROT == kWhole ? 0 : i] * sn;
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c[e] = 1.f;
        s[e] = 0.f;
      }
    }
  }
  // The zeros behind the pieces of the wave's rows.
  __device__ __forceinline__ static void clear(u32x4* rows, int n, int lane) {
    if (D != 96 && lane < n * Shape<D>::tokens) rows[lane * Shape<D>::pitch + Shape<D>::none] = u32x4{0u, 0u, 0u, 0u};
  }
  // The partners of the lane's 8 values of a row, 0 for those that are not turned: their sine is 0, but an infinity times
  // it is not. `row`: the 16-byte pieces of the wave's rows in LDS; only this wave writes and reads them.
  __device__ __forceinline__ void partners(const u32x4& w, const Floats8& x, u32x4* row, int lane, Floats8& xp) const {
    constexpr int L = Shape<D>::lanes;
    if constexpr (ROT == kNext) {
#pragma unroll
      for (int e = 0; e < 8; ++e) xp[e] = x[e ^ 1];
      if (every) return;
#pragma unroll
      for (int e = 0; e < 8; ++e) xp[e] = e < left ? xp[e] : 0.f;
    } else if constexpr (ROT == kWhole || ROT == kAny) {
      u32x4* mine = row + lane / L * Shape<D>::pitch;
      mine[lane % L] = w;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if constexpr (ROT == kWhole) {
        widen(mine[from[0]], xp);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          xp[e] = __uint_as_float((uint32_t) * reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(mine) + from[e]) << 16);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) xp[e] = 0.f;
    }
  }
};

// w[e], e = 8 l .. 8 l + 7, or `none` where there is no array. Lanes behind the row read its last values.
template <int D>
__device__ __forceinline__ void load8(const float* w, int l, float none, Floats8& x) {
  const int e0 = min(8 * l, D - 8);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = w ? w[e0 + e] : none;
}
// The same of the values' partners, 0 for values that are not turned. (kAny: only where there is no array; with one they come
// from LDS.)
template <int D, int ROT>
__device__ __forceinline__ void load_partners(const float* w, int l, float none, const Turns<D, ROT>& t, Floats8& x) {
  if constexpr (ROT == kNext) {
    Floats8 own;
    load8<D>(w, l, none, own);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < t.left ? own[e ^ 1] : 0.f;
  } else if constexpr (ROT == kWhole) {
    load8<D>(w, t.from[0], none, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = t.from[0] < Shape<D>::none ? x[e] : 0.f;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = ROT == kAny ? none : 0.f;
  }
}

// x less its mean (kLayer), and the factor that norms it. A lane behind the row holds zeros and keeps them.
template <int D, int NORM>
__device__ __forceinline__ float norm_factor(float eps, bool in_row, Floats8& x, float& mean) {
  mean = 0.f;
  if constexpr (NORM == kNone) return 1.f;
  if constexpr (NORM == kLayer) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += x[e];
    mean = row_sum<D>(sum) * (1.f / D);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = in_row ? x[e] - mean : 0.f;
  }
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
  return __builtin_amdgcn_rsqf(fmaf(row_sum<D>(sum), 1.f / D, eps));
}

// A lane's token.
struct Token {
  int b, t;
  bool have;   // there is such a token
  bool valid;  // and it is no padding
  bool any;    // so is that of some lane of the wave
  __device__ __forceinline__ Token(const RopeArgs& a, int64_t i) {
    const int64_t total = (int64_t)a.B * a.S;
    have = i < total;
    const uint32_t n = (uint32_t)(have ? i : total - 1);
    b = (int)(n / (uint32_t)a.S);
    t = (int)(n - (uint32_t)b * (uint32_t)a.S);
    valid = have && t < (a.lens ? a.lens[b] : a.S);
    any = __builtin_amdgcn_ballot_w64(valid) != 0;
  }
};

// Forward. Bound by the bytes, each read and written once: 86400 tokens, 72 heads of 96 (93 frames of 720p), 485 us for 2.39 GB, 4.9
// TB/s (a large copy 4.9 to 5.1); 17776 tokens, 144 heads of 64, layer norms, 132 us, 4.95 TB/s. Single tokens by their chain of
// loads: 32 of them, 48 heads of 128, 4.8 us. Four rows of a lane are read together, the next four meanwhile; without
// the next ones two together took 504 us and one 556. Results past the caches: 480, not worth a second kernel.
// With pairs anywhere in the row a workgroup forms the places, and puts the weights, into LDS first: 62982 tokens, 9 heads of 96
// 56 us (places by every lane for its 8 values 70, weights from memory 60); 8 tokens, 10 heads of 64 4.4 us (5.3). Few heads pay for
// a token's angles and a workgroup's places: 60000 tokens, 3 heads of 64 20.9 us for 9.2 us of bytes (19.0 with pieces of 8).
constexpr int kAhead = 4;

template <int D, int NORM, int ROT>
__global__ __launch_bounds__(64 * kRopeWaves) void head_rope_kernel(const RopeArgs a) {
  constexpr int L = Shape<D>::lanes, kTokens = Shape<D>::tokens, kPieces = Shape<D>::pieces;
  __shared__ u32x4 s_rows[ROT >= kWhole ? kRopeWaves * kAhead * kPieces : 1];
  __shared__ PlaceEntry s_place[ROT == kAny ? D : 1];
  // Of q and k: weights, biases, each with the partner's of a value that is not turned, 0, behind it.
  constexpr int kPitch = D + 1;
  __shared__ float s_weights[2][ROT == kAny && NORM != kNone ? 2 * kPitch : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l = lane % L;
  const bool in_row = 8 * l < D;
  const int64_t token0 = ((int64_t)blockIdx.x * kRopeWaves + wave) * kTokens;
  const bool none = token0 >= (int64_t)a.B * a.S;
  if (ROT != kAny && none) return;
  const Token tok(a, token0 + lane / L);
  const bool writes = tok.have && in_row;
  const int at = in_row ? 8 * l : D - 8;  // lanes behind a row read its last values, as zeros
  u32x4* rows = s_rows + (ROT >= kWhole ? wave * kAhead * kPieces : 0);

  // Heads of q, k and v in a line; this wave's are first .. last - 1. A step takes up to kAhead heads of one kind,
  // and the next step's rows are on their way meanwhile (the first one's while the angles are formed).
  const int k0 = a.heads[0], v0 = k0 + a.heads[1], all = v0 + a.heads[2];
  const int first = blockIdx.y * a.heads_per, last = min(first + a.heads_per, all);
  auto kind_of = [&](int f) { return f < k0 ? 0 : f < v0 ? 1 : 2; };
  auto start_of = [&](int kind) { return kind == 0 ? 0 : kind == 1 ? k0 : v0; };
  auto stop = [&](int f) { return min(min(f + kAhead, last), f < k0 ? k0 : f < v0 ? v0 : all); };
  auto load = [&](int f, u32x4 (&in)[kAhead]) {
    const int kind = kind_of(f), h = f - start_of(kind), n = stop(f) - f;
    const Rows x = a.x[kind];
    const uint16_t* x0 = x.p + tok.b * x.batch + tok.t * x.token + h * x.head + at;
    if (tok.any) {  // (all of a step's loads without a branch between them: the last row again where there are fewer)
#pragma unroll
      for (int u = 0; u < kAhead; ++u) in[u] = load16(x0 + min(u, n - 1) * x.head);
    }
    const bool reads = tok.valid && in_row;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) in[u] = reads ? in[u] : u32x4{0u, 0u, 0u, 0u};
  };
  u32x4 in[kAhead], next[kAhead];
  load(first, in);

  Turns<D, ROT> turns;
  if constexpr (ROT == kAny && NORM != kNone) {
    for (int i = threadIdx.x; i < 2 * kPitch; i += 64 * kRopeWaves) {
      const int kind = i / kPitch, e = i % kPitch;
      s_weights[kind][e] = e == D ? 0.f : a.weight[kind] ? a.weight[kind][e] : 1.f;
      if (NORM == kLayer) s_weights[kind][kPitch + e] = e == D || !a.bias[kind] ? 0.f : a.bias[kind][e];
    }
  }
  turns.place(a, l, s_place);
  if (none) return;
  if constexpr (ROT >= kWhole) turns.clear(rows, kAhead, lane);
  // y_e = r (x_e A_e + x_partner B_e) + C_e with x less its mean; A, B and C of the kind `ready`, its weights and
  // biases times the token's cosines and sines.
  Floats8 A, Bp, C, w, wp, bs, bp;
  auto weights = [&](int kind) {
    if constexpr (ROT == kAny && NORM != kNone) {  // (lanes behind the row: signs of 0)
      const float* of = s_weights[kind];
      const int e0 = min(8 * l, D - 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = of[e0 + e];
        wp[e] = of[turns.from[e] / 2];
        bs[e] = NORM == kLayer ? of[kPitch + e0 + e] : 0.f;
        bp[e] = NORM == kLayer ? of[kPitch + turns.from[e] / 2] : 0.f;
      }
      return;
    }
    const float* weight = NORM == kNone ? nullptr : a.weight[kind];
    const float* bias = NORM == kLayer ? a.bias[kind] : nullptr;
    load8<D>(weight, l, 1.f, w);
    load_partners<D, ROT>(weight, l, 1.f, turns, wp);
    load8<D>(bias, l, 0.f, bs);
    load_partners<D, ROT>(bias, l, 0.f, turns, bp);
  };
  int ready = kind_of(first);
  if (ready < 2) weights(ready);
  Floats8 c, s;
  turns.at(a, tok.b, tok.t, c, s);
  auto factors = [&]() {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      A[e] = w[e] * c[e];
      Bp[e] = wp[e] * s[e];
      C[e] = NORM == kLayer ? fmaf(bs[e], c[e], bp[e] * s[e]) : 0.f;
    }
  };
  if (ready < 2) factors();
  const int64_t plane = (int64_t)a.S * D;
  for (int f = first; f < last;) {
    const int f1 = stop(f), kind = kind_of(f);
    if (f1 < last) load(f1, next);
    if (kind < 2 && kind != ready) {
      ready = kind;
      weights(kind);
      factors();
    }
    uint16_t* y0 = a.y[kind] + (((int64_t)tok.b * a.heads[kind] + (f - start_of(kind))) * a.S + tok.t) * D + 8 * l;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (f + u >= f1) break;
      u32x4 out = in[u];
      if (kind < 2 && (NORM != kNone || ROT != kStill)) {
        Floats8 x, xp, y;
        widen(in[u], x);
        turns.partners(in[u], x, rows + (ROT >= kWhole ? kPieces * u : 0), lane, xp);
        float mean;
        const float r = norm_factor<D, NORM>(a.eps, in_row, x, mean);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = ROT == kStill ? x[e] * A[e] : fmaf(x[e], A[e], (NORM == kLayer ? xp[e] - mean : xp[e]) * Bp[e]);
          y[e] = NORM == kNone ? z : NORM == kRms ? r * z : fmaf(r, z, C[e]);
        }
        out = narrow(y);
        if (!tok.valid) out = u32x4{0u, 0u, 0u, 0u};
      }
      if (writes) *reinterpret_cast<u32x4*>(y0 + u * plane) = out;
    }
    if constexpr (ROT >= kWhole) {  // the rows in LDS are read before the next ones replace them
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) in[u] = next[u];
    f = f1;
  }
}

// Gradients. With g the gradient of a row turned back, xhat the normed row before weights:
//   db = sum g,  dw = sum g xhat,  u = g w,  dx = r (u - [mean u] - xhat mean(u xhat)).
// Bound by the bytes: 28800 tokens, 72 heads of 96, 229 us for 1.19 GB (5.2 TB/s). The row is read behind the store of the one
// before it: reading it earlier, beside that one's work, took 261 us, two rows at a time 357.
// Workgroups first[kind] .. first[kind + 1] - 1 have the rows of q, k or v and deal out (tokens, heads) items among
// their waves, so that the sums of weights and biases, kept in a lane's registers, leave few rows of partial
// sums; they are added in an order that the sizes set. After kChain rows a lane's sums go to LDS and start again, so that no
// chain of additions grows with the call: 86400 tokens, 24 + 24 heads, have 344 rows a lane. (Four waves a SIMD unit, the workgroups
// that are resident at once: without that bound layer norms with pairs anywhere take 130 registers, and 62982 tokens, 9 heads of 96,
// 107 us for 75.)
constexpr int kChain = 256;
template <int D, int NORM, int ROT>
__global__ __launch_bounds__(64 * kRopeWaves, 4) void head_rope_grad_kernel(const RopeArgs a) {
  constexpr int L = Shape<D>::lanes, kTokens = Shape<D>::tokens;
  __shared__ u32x4 s_rows[ROT >= kWhole ? kRopeWaves * Shape<D>::pieces : 1];
  __shared__ PlaceEntry s_place[ROT == kAny ? D : 1];
  __shared__ float s_sum[kRopeWaves][2][D];
  __shared__ float s_run[NORM == kLayer ? 16 : NORM != kNone ? 8 : 1][64 * kRopeWaves];  // a lane's sums of earlier chains
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l = lane % L;
  const bool in_row = 8 * l < D;
  const int kind = (int)blockIdx.x < a.first[1] ? 0 : (int)blockIdx.x < a.first[2] ? 1 : 2;
  const int waves = (a.first[kind + 1] - a.first[kind]) * kRopeWaves;
  const int groups = (int)(((int64_t)a.B * a.S + kTokens - 1) / kTokens);
  const int heads = a.heads[kind], parts = (heads + a.heads_per - 1) / a.heads_per;
  const int64_t items = (int64_t)groups * parts, plane = (int64_t)a.S * D;
  const bool normed = NORM != kNone && kind < 2, turned = ROT != kStill && kind < 2;
  u32x4* rows = s_rows + (ROT >= kWhole ? wave * Shape<D>::pieces : 0);
  const int at = 8 * l;
  const Rows x = a.x[kind], dx = a.dx[kind];

  Turns<D, ROT> turns;
  Floats8 w, dw, db;
  if (kind < 2) {
    turns.place(a, l, s_place);
    if constexpr (ROT >= kWhole) turns.clear(rows, 1, lane);
    load8<D>(NORM == kNone ? nullptr : a.weight[kind], l, 1.f, w);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[e] = db[e] = 0.f;
  int chain = 0;  // rows in dw and db
  bool runs = false;
  for (int64_t item = (int64_t)((int)blockIdx.x - a.first[kind]) * kRopeWaves + wave; item < items; item += waves) {
    const int part = (int)(item / groups);
    const Token tok(a, (item - (int64_t)part * groups) * kTokens + lane / L);
    const bool reads = tok.valid && in_row, writes = tok.have && in_row;
    const int h0 = part * a.heads_per, h1 = min(h0 + a.heads_per, heads);
    const uint16_t* g0 = a.y[kind] + ((int64_t)tok.b * heads * a.S + tok.t) * D + at;
    const uint16_t* x0 = x.p + tok.b * x.batch + tok.t * x.token + at;
    uint16_t* d0 = dx.p + tok.b * dx.batch + tok.t * dx.token + at;
    u32x4 xin = {0u, 0u, 0u, 0u}, gin = {0u, 0u, 0u, 0u};
    auto load = [&](int h, u32x4& xr, u32x4& g) {
      if (reads) {
        g = load16(g0 + h * plane);
        if (normed) xr = load16(x0 + h * x.head);
      }
    };
    load(h0, xin, gin);
    Floats8 c, s;
    if (turned) turns.at(a, tok.b, tok.t, c, s);
    for (int h = h0; h < h1; ++h) {
      u32x4 out = gin;
      if (normed || turned) {
        Floats8 g;
        widen(gin, g);
        if (turned) {
          Floats8 gp;
          turns.partners(gin, g, rows, lane, gp);
#pragma unroll
          for (int e = 0; e < 8; ++e) gp[e] *= s[e];
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = fmaf(g[e], c[e], -gp[e]);
          if constexpr (ROT >= kWhole) {  // the row in LDS is read before the next one replaces it
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
          }
        }
        if constexpr (NORM != kNone) {
          Floats8 x;
          widen(xin, x);
          float mean;
          const float r = norm_factor<D, NORM>(a.eps, in_row, x, mean);
          float along = 0.f, sum = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] *= r;
            dw[e] = fmaf(g[e], x[e], dw[e]);
            if constexpr (NORM == kLayer) db[e] += g[e];
            g[e] *= w[e];
            along = fmaf(g[e], x[e], along);
            sum += g[e];
          }
          along = row_sum<D>(along) * (1.f / D);
          sum = NORM == kLayer ? row_sum<D>(sum) * (1.f / D) : 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = r * (fmaf(-x[e], along, g[e]) - sum);
        }
        out = narrow(g);
        if (!tok.valid) out = u32x4{0u, 0u, 0u, 0u};
      }
      if (writes) *reinterpret_cast<u32x4*>(d0 + h * dx.head) = out;
      if (h + 1 < h1) load(h + 1, xin, gin);
    }
    chain += h1 - h0;
    if (normed && chain + a.heads_per > kChain) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s_run[e][threadIdx.x] = runs ? s_run[e][threadIdx.x] + dw[e] : dw[e];
        dw[e] = 0.f;
        if constexpr (NORM == kLayer) {
          s_run[8 + e][threadIdx.x] = runs ? s_run[8 + e][threadIdx.x] + db[e] : db[e];
          db[e] = 0.f;
        }
      }
      chain = 0;
      runs = true;
    }
  }
  if constexpr (NORM != kNone) {
    if (kind < 2 && a.part) {
      if (runs) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dw[e] += s_run[e][threadIdx.x];
          if constexpr (NORM == kLayer) db[e] += s_run[8 + e][threadIdx.x];
        }
      }
      // Tokens of the wave, then waves, then (the second kernel) workgroups.
#pragma unroll
      for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int m = L; m < 64; m <<= 1) {
          dw[e] += __shfl_xor(dw[e], m);
          if constexpr (NORM == kLayer) db[e] += __shfl_xor(db[e], m);
        }
        if (lane < L && in_row) {
          s_sum[wave][0][8 * l + e] = dw[e];
          if constexpr (NORM == kLayer) s_sum[wave][1][8 * l + e] = db[e];
        }
      }
      __syncthreads();
      for (int i = threadIdx.x; i < (NORM == kLayer ? 2 : 1) * D; i += 64 * kRopeWaves) {
        float sum = 0.f;
#pragma unroll
        for (int x = 0; x < kRopeWaves; ++x) sum += s_sum[x][i / D][i % D];
        a.part[(int64_t)blockIdx.x * 2 * D + i] = sum;
      }
    }
  }
}

// Adds the workgroups' partial sums: a workgroup per 16 columns of one of the four sums (q's weight and bias,
// k's).
constexpr int kSumColumns = 16, kSumThreads = 256;
__global__ __launch_bounds__(kSumThreads) void head_rope_sum_kernel(const RopeArgs a) {
  constexpr int kSlices = kSumThreads / kSumColumns;
  __shared__ float s_sum[kSlices][kSumColumns];
  float* out = a.sum[blockIdx.y];
  if (!out) return;
  const int kind = blockIdx.y / 2;
  const int col = threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns;
  const int e = blockIdx.x * kSumColumns + col;
  float sum = 0.f;
#pragma unroll 8
  for (int w = a.first[kind] + slice; w < a.first[kind + 1]; w += kSlices)
    sum += a.part[((int64_t)w * 2 + blockIdx.y % 2) * a.d + e];
  s_sum[slice][col] = sum;
  __syncthreads();
  if (slice == 0) {
    sum = 0.f;
#pragma unroll
    for (int x = 0; x < kSlices; ++x) sum += s_sum[x][col];
    out[e] = sum;
  }
}

template <int D, int NORM, int ROT>
hipError_t run(const RopeArgs& a, bool grad, hipStream_t s) {
  if (grad) {
    head_rope_grad_kernel<D, NORM, ROT><<<(unsigned)a.first[3], 64 * kRopeWaves, 0, s>>>(a);
    if (NORM != kNone && a.part) head_rope_sum_kernel<<<dim3((unsigned)(D / kSumColumns), 4), kSumThreads, 0, s>>>(a);
  } else {
    const int64_t waves = ((int64_t)a.B * a.S + Shape<D>::tokens - 1) / Shape<D>::tokens;
    const int heads = a.heads[0] + a.heads[1] + a.heads[2];
    const dim3 grid((unsigned)((waves + kRopeWaves - 1) / kRopeWaves), (unsigned)((heads + a.heads_per - 1) / a.heads_per));
    head_rope_kernel<D, NORM, ROT><<<grid, 64 * kRopeWaves, 0, s>>>(a);
  }
  return hipGetLastError();
}
template <int D, int NORM>
hipError_t run_rot(const RopeArgs& a, bool grad, hipStream_t s) {
  if (a.layout == 0) return run<D, NORM, kStill>(a, grad, s);
  if (a.layout == 1) return run<D, NORM, kNext>(a, grad, s);
  return a.whole ? run<D, NORM, kWhole>(a, grad, s) : run<D, NORM, kAny>(a, grad, s);
}
template <int D>
hipError_t run_norm(const RopeArgs& a, bool grad, hipStream_t s) {
  if (a.norm == kNone) return run_rot<D, kNone>(a, grad, s);
  return a.norm == kRms ? run_rot<D, kRms>(a, grad, s) : run_rot<D, kLayer>(a, grad, s);
}
hipError_t run_all(const RopeArgs& a, bool grad, hipStream_t s) {
  if (a.d == 64) return run_norm<64>(a, grad, s);
  return a.d == 96 ? run_norm<96>(a, grad, s) : run_norm<128>(a, grad, s);
}

}  // namespace

hipError_t launch_head_rope(const RopeArgs& a, hipStream_t stream) { return run_all(a, false, stream); }
hipError_t launch_head_rope_grad(const RopeArgs& a, hipStream_t stream) { return run_all(a, true, stream); }

}  // namespace ta
