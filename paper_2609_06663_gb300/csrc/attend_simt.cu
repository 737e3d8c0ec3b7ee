// Attention of the decode step on CUDA cores: fp32 tensors, and bf16 ones with
// ECOKV_FLAG_FORCE_SIMT.  Items and tiles as in attend.cuh.
//
// Items of up to 32 rows (a decode step's own keys, a small batch's prefix): each warp
// has sixteen keys of a tile and all of the rows, with a maximum, sum and output of
// its own that are joined at the item's end.  K and V go from memory to registers
// once: lanes 2k and 2k + 1 share the dot products of key k, then lane c has columns
// 4c .. 4c + 3 of the sixteen rows of V.  Bound by those loads: the next tile's K is
// on its way from the moment that this one's last scores are there.  The loop over
// rows stays rolled, its sums in shared memory: a call of a few tiles runs its code
// but once, and fetching code takes longer than running it (8 heads: 8 sequences of up
// to three tokens over 128 rows 16.5 us, unrolled for eight rows with the sums in
// registers 22.2; 13 single tokens over 1369 rows and up to 1252 of their own 40.3 and
// 89).  A row is one chain of products, shuffles and exponential behind the other, and
// a tile takes as long as its rows do, which the dealing does not count.
//
// Items of more rows, in groups of 64: a CTA of 256 threads holds an item's queries, a
// tile of 128 keys and its values in shared memory as fp32 (82 tokens of 8 sequences, 28
// heads over 4, 1369 rows and up to 300 of their own: 93 us, 19 TFLOP/s).  Thread (ty, tx)
// of 16 x 16 forms the scores of its rows ty R .. ty R + R - 1 with the keys tx + 16 j, a
// row's maximum and sum are four shuffles away, and the same thread then sums columns
// 4 tx .. and 64 + 4 tx .. of its rows' outputs over the tile, which stay in registers
// through the item.

#include <math.h>

#include <atomic>

#include "attend.cuh"
#include "decode_ptx.cuh"

namespace ecokv {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64;    // rows a row tile
constexpr int kPad = kD + 4; // floats a padded row: 16-byte reads of 8 consecutive rows meet all banks

struct Smem {
  float q[kRows][kPad];
  float k[kKeys][kPad];
  float v[kKeys][kD];   // (k and v follow each other: 32 rows of 8 warps of the items of few rows)
  float p[kRows][kPad];
  int64_t at[2][kKeys];  // where the keys of this tile and the next are, see key_offset
  struct {               // of the items of few rows, a warp's maxima and sums by row, and a row's weights
    float m[8][32], l[8][32];
    __align__(16) float p[8][16];
  } few;
  Item item;
  int more;
};
static_assert(sizeof(float) * kKeys * (kPad + kD) >= sizeof(float) * 8 * 32 * kD, "outputs of the items of few rows");
static_assert(sizeof(Smem) <= 232448, "one CTA's shared memory");

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xffff0000u));
}

// Offset of key j of the item in K and V, negative: none (a page number out of range).
__device__ __forceinline__ int64_t key_offset(const AttendArgs& a, const Item& it, int j) {
  if (it.source == 0) {
    const int64_t r = (int64_t)it.row0 + j;
    return (a.prefix.head_off ? 0 : (int64_t)it.head * a.prefix.head_stride) + r * a.prefix.row_stride;
  }
  const int page = a.cache.table[(int64_t)it.seq * a.cache.table_stride + (j >> a.page_shift)];
  if (page < 0 || page >= a.cache.n_pages) {
    note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)it.seq);
    return -1;
  }
  return (int64_t)page * a.cache.page_stride + (int64_t)it.head * a.cache.head_stride +
         (int64_t)(j & (a.cache.page_size - 1)) * a.cache.slot_stride;
}

constexpr int kFew = 32;              // rows of an item whose keys are split between the warps
constexpr int kWarps = kThreads / 32;
constexpr int kOwn = kKeys / kWarps;  // keys of a tile that a warp has

template <typename T>
__device__ __forceinline__ void item_few(const AttendArgs& a, Smem& s, const Item& it) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, kk = lane >> 1, half = lane & 1;
  const int rows = it.ntok * a.g;
  // in the place of K and V: outputs [warp][row][d]; maxima and sums [warp][row]
  float* out = &s.k[0][0] + warp * kFew * kD;
  float* mx = s.few.m[warp];
  float* sum = s.few.l[warp];
  float* pw = s.few.p[warp];
#pragma unroll 1
  for (int r = warp; r < rows; r += kWarps) {
    const int k = r / a.g;
    *reinterpret_cast<float4*>(&s.q[r][lane * 4]) =
        load4(static_cast<const T*>(a.q) + (int64_t)(it.tok0 + k) * a.q_token +
              (int64_t)(it.head * a.g + r - k * a.g) * a.q_head + lane * 4);
  }
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    *reinterpret_cast<float4*>(out + r * kD + lane * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
    if (lane == 0) {
      mx[r] = -INFINITY;
      sum[r] = 0.f;
    }
  }
  const T* K = static_cast<const T*>(it.source == 0 ? a.prefix.k : a.cache.k);
  const T* V = static_cast<const T*>(it.source == 0 ? a.prefix.v : a.cache.v);
  const int t1 = it.tile0 + it.ntiles;
  float4 kr[kOwn], vr[kOwn];
  int64_t at = -1;  // of this lane pair's key
  __syncthreads();
#pragma unroll 1
  for (int t = it.tile0; t < t1; ++t) {
    const int j = t * kKeys + warp * kOwn + kk;
    if (t == it.tile0) at = j < it.vis ? key_offset(a, it, j) : -1;
    if (t == it.tile0) {
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {  // (every other 16 bytes of the row, its neighbour lane the others)
        kr[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at >= 0) kr[i] = load4(K + at + (2 * i + half) * 4);
      }
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int64_t o = __shfl_sync(0xffffffffu, (long long)at, 2 * i);
      vr[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (o >= 0) vr[i] = load4(V + o + lane * 4);
    }
    int64_t next = -1;
    if (t + 1 < t1 && j + kKeys < it.vis) next = key_offset(a, it, j + kKeys);
#pragma unroll 1
    for (int r = 0; r < rows; ++r) {
      float e = 0.f, f = 0.f;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const float4 q4 = *reinterpret_cast<const float4*>(&s.q[r][(2 * i + half) * 4]);
        e = fmaf(q4.x, kr[i].x, e);
        f = fmaf(q4.y, kr[i].y, f);
        e = fmaf(q4.z, kr[i].z, e);
        f = fmaf(q4.w, kr[i].w, f);
      }
      e += f;
      e += __shfl_xor_sync(0xffffffffu, e, 1);
      if (r == rows - 1 && t + 1 < t1) {
        at = next;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          kr[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (at >= 0) kr[i] = load4(K + at + (2 * i + half) * 4);
        }
      }
      const float y = j < it.lim0 + r / a.g * it.slope ? e * a.scale_log2 : -INFINITY;
      const float m = mx[r], mn = fmaxf(m, ptx::redux_max(y)), ref = mn == -INFINITY ? 0.f : mn;
      const float corr = ptx::ex2(m - ref);
      float l = sum[r] * corr;
      if (half == 0) pw[kk] = ptx::ex2(y - ref);
      float4 o = *reinterpret_cast<const float4*>(out + r * kD + lane * 4);
      o.x *= corr;
      o.y *= corr;
      o.z *= corr;
      o.w *= corr;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kOwn; i += 4) {
        const float4 p4 = *reinterpret_cast<const float4*>(pw + i);
        const float p[4] = {p4.x, p4.y, p4.z, p4.w};
        l += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          o.x = fmaf(p[k], vr[i + k].x, o.x);
          o.y = fmaf(p[k], vr[i + k].y, o.y);
          o.z = fmaf(p[k], vr[i + k].z, o.z);
          o.w = fmaf(p[k], vr[i + k].w, o.w);
        }
      }
      *reinterpret_cast<float4*>(out + r * kD + lane * 4) = o;
      if (lane == 0) {  // (ahead of the barrier: an item of one row reads them next, a tile on)
        mx[r] = mn;
        sum[r] = l;
      }
      __syncwarp();
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int r = warp; r < rows; r += kWarps) {  // the warps' sums, a warp a row
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s.few.m[w][r]);
    const float ref = M == -INFINITY ? 0.f : M;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float c = ptx::ex2(s.few.m[w][r] - ref);
      const float4 v = *reinterpret_cast<const float4*>(&s.k[0][0] + (w * kFew + r) * kD + lane * 4);
      L = fmaf(c, s.few.l[w][r], L);
      acc.x = fmaf(c, v.x, acc.x);
      acc.y = fmaf(c, v.y, acc.y);
      acc.z = fmaf(c, v.z, acc.z);
      acc.w = fmaf(c, v.w, acc.w);
    }
    const int k = r / a.g;
    const bool first = it.tile0 == 0;
    const size_t to = first ? first_row(a, it.source, it.tok0 + k, it.head * a.g + r - k * a.g)
                            : next_row(a, blockIdx.x, 0, r);
    *reinterpret_cast<float4*>((first ? a.first_o : a.next_o) + to * kD + lane * 4) = acc;
    if (lane == 0) (first ? a.first_ml : a.next_ml)[to] = make_float2(M, L);
  }
}

template <typename T>
__device__ __forceinline__ void item_rows(const AttendArgs& a, Smem& s, const Item& it) {
  constexpr int R = kRows / 16;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 31, warp = tid >> 5;
  const int rows = it.ntok * a.g;
  // queries
  for (int r = warp; r < 16 * R; r += kThreads / 32) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows) {
      const int k = r / a.g;
      v = load4(static_cast<const T*>(a.q) + (int64_t)(it.tok0 + k) * a.q_token +
                (int64_t)(it.head * a.g + r - k * a.g) * a.q_head + lane * 4);
    }
    *reinterpret_cast<float4*>(&s.q[r][lane * 4]) = v;
  }
  float m[R], l[R], o[R][8];
  int lim[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
    lim[r] = it.lim0 + (ty * R + r) / a.g * it.slope;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[r][c] = 0.f;
  }
  const T* K = static_cast<const T*>(it.source == 0 ? a.prefix.k : a.cache.k);
  const T* V = static_cast<const T*>(it.source == 0 ? a.prefix.v : a.cache.v);
  auto look_up = [&](int t) {  // a tile ahead, so that its rows' reads do not wait for page numbers
    const int j = t * kKeys + tid;
    if (tid < kKeys) s.at[t & 1][tid] = j < it.vis ? key_offset(a, it, j) : -1;
  };
  look_up(it.tile0);
  for (int t = it.tile0; t < it.tile0 + it.ntiles; ++t) {
    __syncthreads();
#pragma unroll 8
    for (int i = 0; i < kKeys / (kThreads / 32); ++i) {
      const int kk = warp + i * (kThreads / 32);
      const int64_t at = s.at[t & 1][kk];
      float4 k4 = make_float4(0.f, 0.f, 0.f, 0.f), v4 = k4;
      if (at >= 0) {
        k4 = load4(K + at + lane * 4);
        v4 = load4(V + at + lane * 4);
      }
      *reinterpret_cast<float4*>(&s.k[kk][lane * 4]) = k4;
      *reinterpret_cast<float4*>(&s.v[kk][lane * 4]) = v4;
    }
    if (t + 1 < it.tile0 + it.ntiles) look_up(t + 1);
    __syncthreads();
    const int nv = min(it.vis - t * kKeys, kKeys), nc = (nv + 15) >> 4;  // keys that are there, in sixteens
    float x[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < 8; ++c) x[r][c] = 0.f;
#pragma unroll 1
    for (int e = 0; e < kD; e += 4) {
      float4 q4[R];
#pragma unroll
      for (int r = 0; r < R; ++r) q4[r] = *reinterpret_cast<const float4*>(&s.q[ty * R + r][e]);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        if (c >= nc) break;
        const float4 k4 = *reinterpret_cast<const float4*>(&s.k[tx + 16 * c][e]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          x[r][c] = fmaf(q4[r].x, k4.x, x[r][c]);
          x[r][c] = fmaf(q4[r].y, k4.y, x[r][c]);
          x[r][c] = fmaf(q4[r].z, k4.z, x[r][c]);
          x[r][c] = fmaf(q4[r].w, k4.w, x[r][c]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        x[r][c] = t * kKeys + tx + 16 * c < lim[r] ? x[r][c] * a.scale_log2 : -INFINITY;
        mx = fmaxf(mx, x[r][c]);
      }
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
      const float mn = fmaxf(m[r], mx), ref = mn == -INFINITY ? 0.f : mn;
      const float corr = ptx::ex2(m[r] - ref);
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float p = ptx::ex2(x[r][c] - ref);
        sum += p;
        s.p[ty * R + r][tx + 16 * c] = p;
      }
      l[r] = fmaf(l[r], corr, sum);  // this thread's share of the row's sum
      m[r] = mn;
#pragma unroll
      for (int c = 0; c < 8; ++c) o[r][c] *= corr;
    }
    __syncwarp();  // (a row's sixteen threads are in one warp)
#pragma unroll 1
    for (int k0 = 0; k0 < nv; k0 += 4) {
      float4 p4[R];
#pragma unroll
      for (int r = 0; r < R; ++r) p4[r] = *reinterpret_cast<const float4*>(&s.p[ty * R + r][k0]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 va = *reinterpret_cast<const float4*>(&s.v[k0 + k][4 * tx]);
        const float4 vb = *reinterpret_cast<const float4*>(&s.v[k0 + k][64 + 4 * tx]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float p = k == 0 ? p4[r].x : k == 1 ? p4[r].y : k == 2 ? p4[r].z : p4[r].w;
          o[r][0] = fmaf(p, va.x, o[r][0]);
          o[r][1] = fmaf(p, va.y, o[r][1]);
          o[r][2] = fmaf(p, va.z, o[r][2]);
          o[r][3] = fmaf(p, va.w, o[r][3]);
          o[r][4] = fmaf(p, vb.x, o[r][4]);
          o[r][5] = fmaf(p, vb.y, o[r][5]);
          o[r][6] = fmaf(p, vb.z, o[r][6]);
          o[r][7] = fmaf(p, vb.w, o[r][7]);
        }
      }
    }
    __syncwarp();
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
    const int row = ty * R + r;
    if (row < rows) {
      const int k = row / a.g;
      const bool first = it.tile0 == 0;
      const size_t at = first ? first_row(a, it.source, it.tok0 + k, it.head * a.g + row - k * a.g)
                              : next_row(a, blockIdx.x, 0, row);
      float* dst = (first ? a.first_o : a.next_o) + at * kD;
      *reinterpret_cast<float4*>(dst + 4 * tx) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
      *reinterpret_cast<float4*>(dst + 64 + 4 * tx) = make_float4(o[r][4], o[r][5], o[r][6], o[r][7]);
      if (tx == 0) (first ? a.first_ml : a.next_ml)[at] = make_float2(m[r], l[r]);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 1) attend_simt_kernel(const __grid_constant__ AttendArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Smem& s = *reinterpret_cast<Smem*>(smem_raw);
  const int lane = threadIdx.x & 31;
  ptx::grid_wait();
  Walk w;
  if (threadIdx.x < 32) w.begin(a, blockIdx.x, lane);
  while (true) {
    __syncthreads();
    if (threadIdx.x < 32) {
      Item it;
      const bool more = w.next(a, it);
      if (lane == 0) {
        s.item = it;
        s.more = more ? 1 : 0;
      }
    }
    __syncthreads();
    if (s.more == 0) break;
    const Item it = s.item;
    if (it.ntok * a.g <= kFew) item_few<T>(a, s, it);
    else item_rows<T>(a, s, it);
  }
  ptx::grid_trigger();
}

template <typename T>
cudaError_t launch(const AttendArgs& a, cudaStream_t st) {
  static std::atomic<bool> set[64];  // a racing thread repeats the idempotent setting
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!set[dev].load()) {
    e = cudaFuncSetAttribute(attend_simt_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
    if (e != cudaSuccess) return e;
    set[dev].store(true);
  }
  return launch_behind(attend_simt_kernel<T>, (unsigned)a.P, kThreads, sizeof(Smem), st, a);
}

}  // namespace

cudaError_t launch_attend_simt(const AttendArgs& a, ecokv_dtype dt, cudaStream_t st) {
  return dt == ECOKV_F32 ? launch<float>(a, st) : launch<__nv_bfloat16>(a, st);
}

}  // namespace ecokv
