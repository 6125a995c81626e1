// Argument checks shared by the C-ABI translation units whose workspaces are the caller's.
#pragma once
#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>
#include <initializer_list>
#include <string>

#include "host_internal.h"
#include "tile_attn.h"

namespace ta {
namespace host {

// Workgroups that the device runs at a time at two per compute unit (256 units). Work is cut by
// this number, not by the device's own, so that workspaces have the same size everywhere.
constexpr int64_t kSlots = 512;
constexpr int64_t kMaxGrid = (int64_t)UINT32_MAX / 256 - 8;

// Results of more bytes than this leave past the caches: half of the last level.
constexpr size_t kStaysInCache = (size_t)128 << 20;

struct Span {
  const void* p;
  size_t bytes;
};
inline size_t bf16s(int64_t n) { return (size_t)n * 2; }

inline int check_aligned(std::initializer_list<const void*> ps, unsigned align, const char* what) {
  for (const void* p : ps)
    if (p && reinterpret_cast<uintptr_t>(p) % align) return fail(TA_ERR_ALIGN, what);
  return TA_OK;
}
// Outputs (and the workspace) must overlap neither an input nor each other.
inline int check_apart(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
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
inline int launched(hipError_t e) {
  if (e != hipSuccess) return fail(TA_ERR_HIP, std::string("kernel launch: ") + hipGetErrorString(e));
  clear_error();
  return TA_OK;
}

inline int check_grid(double workgroups) {
  return workgroups <= (double)kMaxGrid ? TA_OK : fail(TA_ERR_BAD_SHAPE, "the call exceeds the grid limit");
}
inline int check_dim(int d) {
  return d == 64 || d == 96 || d == 128 ? TA_OK : fail(TA_ERR_HEAD_DIM, "d must be 64, 96 or 128");
}

inline int check_workspace(const void* ws, size_t have, size_t need) {
  if (have < need || (need && !ws))
    return fail(TA_ERR_BAD_SHAPE, "the workspace is smaller than the call needs (" + std::to_string(need) + " bytes)");
  return check_aligned({ws}, 16, "the workspace must be 16-byte aligned");
}

}  // namespace host
}  // namespace ta
