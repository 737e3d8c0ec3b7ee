// Rows of a paged cache that move to the front of their sequence, or to another cache
// (drafts.cu, prune.cu).
//
// What bounds it is memory: every row is read and written once, 16 bytes a lane.  In
// one cache a row may lie where another one goes: row i of a list comes from slot
// src(i) >= dst(i) and the sources ascend, so a row that is written over is one that the list
// has passed, or one of those at hand.  A unit (sequence, head, K or V) takes its list
// in chunks, all of a chunk read before any of it is written; with few units a
// cluster of CTAs shares a chunk, its barrier between the two.  Where a chunk's rows are is
// looked up, a thread a row, while those of the chunk before it are on their way.
#pragma once

#include <cooperative_groups.h>

#include "attend.cuh"
#include "decode_ptx.cuh"

namespace ecokv {

constexpr int kMoveBytes = 32 * 1024;  // of a chunk of one CTA

struct MoveArgs {
  ecokv_pages from, to;           // the same pages in one cache
  ecokv_weights w_from, w_to;     // w NULL: none
  int from_shift, to_shift;
  int h_kv, batch;
  int ctas;                       // of a unit
  int cluster;                    // CTAs that wait for each other
  int in_place;
  unsigned* status;               // may be NULL
};

__device__ __forceinline__ void flag(unsigned* status, unsigned detail) {
  if (status != nullptr && atomicCAS(status, 0u, (unsigned)ECOKV_ERR_DEVICE_INDEX) == 0u) status[1] = detail;
}

// Place of a sequence's slot; page -1: out of range.
struct Place {
  int page, row;
};
__device__ __forceinline__ Place place_of(const ecokv_pages& c, int shift, int b, int slot, unsigned* status) {
  Place p;
  p.row = slot & (c.page_size - 1);
  p.page = -1;
  const int col = slot >> shift;
  if (col < c.table_stride) p.page = c.table[(int64_t)b * c.table_stride + col];
  if (p.page < 0 || p.page >= c.n_pages) {
    flag(status, (unsigned)b);
    p.page = -1;
  }
  return p;
}
__device__ __forceinline__ int64_t offset_of(const ecokv_pages& c, Place p, int h) {
  return (int64_t)p.page * c.page_stride + (int64_t)h * c.head_stride + (int64_t)p.row * c.slot_stride;
}
__device__ __forceinline__ int64_t offset_of(const ecokv_weights& w, Place p, int h) {
  return (int64_t)p.page * w.page_stride + (int64_t)h * w.head_stride + (int64_t)p.row * w.slot_stride;
}

// One CTA's share of the rows [i0, n) of unit (b, h, kv): row i from slot src(i) to slot dst0 +
// i.  src: row number -> slot, the same in every CTA.  E: bytes an element.  All of the
// cluster's CTAs call it with the same i0 and n.
template <int E, int kThreads, typename Src>
__device__ __forceinline__ void move_rows(const MoveArgs& a, int b, int h, int kv, int rank, int i0, int n, int dst0,
                                          Src src) {
  constexpr int kLanes = kD * E / 16;               // lanes a row
  constexpr int kAtOnce = kThreads / kLanes;        // rows a step of the CTA
  constexpr int kChunk = kMoveBytes / (kD * E);
  constexpr int kMoveRows = kChunk / kAtOnce;       // rows whose pieces a thread has in flight
  static_assert(kChunk <= kThreads, "a thread a row");
  // bytes from k or v, from and to; from < 0: the row stays.  (Three chunks': while a warp
  // looks the next up, another may still write the one before.)
  __shared__ longlong2 places[3][kChunk];
  const int lane = threadIdx.x % kLanes, r0 = threadIdx.x / kLanes;
  const char* x = static_cast<const char*>(kv == 0 ? a.from.k : a.from.v) + lane * 16;
  char* y = static_cast<char*>(kv == 0 ? a.to.k : a.to.v) + lane * 16;
  const bool weights = kv == 0 && a.w_to.w != nullptr;
  float w = 0.f;
  float* w_at = nullptr;
  auto look_up = [&](int base, int buf) {
    const int i = base + rank * kChunk + (int)threadIdx.x;
    if (threadIdx.x >= kChunk) return;
    longlong2 at = make_longlong2(-1, -1);
    if (weights) w_at = nullptr;
    const int s = i < n ? src(i) : 0;
    if (i < n && !(a.in_place && s == dst0 + i)) {
      const Place p = place_of(a.from, a.from_shift, b, s, a.status);
      const Place q = place_of(a.to, a.to_shift, b, dst0 + i, a.status);
      if (p.page >= 0 && q.page >= 0) {
        at = make_longlong2(offset_of(a.from, p, h) * E, offset_of(a.to, q, h) * E);
        if (weights) {
          w_at = a.w_to.w + offset_of(a.w_to, q, h);
          w = a.w_from.w[offset_of(a.w_from, p, h)];
        }
      }
    }
    places[buf][threadIdx.x] = at;
  };
  if (i0 >= n) return;
  look_up(i0, 0);
  __syncthreads();
  int buf = 0;
#pragma unroll 1
  for (int base = i0; base < n; base += kChunk * a.ctas) {
    const int next = buf == 2 ? 0 : buf + 1;
    uint4 v[kMoveRows];
#pragma unroll
    for (int k = 0; k < kMoveRows; ++k) {
      const int64_t at = places[buf][r0 + k * kAtOnce].x;
      if (at >= 0) v[k] = *reinterpret_cast<const uint4*>(x + at);
    }
    const float w_now = w;
    float* const w_to = w_at;
    if (base + kChunk * a.ctas < n) look_up(base + kChunk * a.ctas, next);
    if (a.in_place && a.cluster > 1) cooperative_groups::this_cluster().sync();
    else __syncthreads();
#pragma unroll
    for (int k = 0; k < kMoveRows; ++k) {
      const longlong2 at = places[buf][r0 + k * kAtOnce];
      if (at.x >= 0) *reinterpret_cast<uint4*>(y + at.y) = v[k];
    }
    if (weights && threadIdx.x < kChunk && w_to != nullptr) *w_to = w_now;
    buf = next;
  }
}

// Launch `kernel` in clusters of a.cluster CTAs.
template <typename... A>
cudaError_t launch_move(void (*kernel)(A...), const MoveArgs& a, unsigned grid, unsigned threads, size_t smem,
                        cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)a.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

inline bool weights_ok(const ecokv_weights* w) {
  return w->w != nullptr && ((uintptr_t)w->w & 3u) == 0 && w->page_stride > 0 && w->head_stride > 0 &&
         w->slot_stride > 0;
}
// Whether n int32 at x and m at y have none in common.
inline bool apart(const void* x, int64_t n, const void* y, int64_t m) {
  const uintptr_t a = (uintptr_t)x, b = (uintptr_t)y;
  return a + (uintptr_t)n * 4 <= b || b + (uintptr_t)m * 4 <= a;
}
// lengths_out is the lengths, or apart from them.
inline bool lengths_ok(const int32_t* lengths, const int32_t* out, int32_t batch) {
  return out != nullptr && ((uintptr_t)out & 3u) == 0 && (out == lengths || apart(lengths, batch, out, batch));
}

}  // namespace ecokv
