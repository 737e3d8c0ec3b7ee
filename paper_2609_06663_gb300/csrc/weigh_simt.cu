// Weights of keys on CUDA cores: fp32 tensors, and bf16 ones with
// ECOKV_FLAG_FORCE_SIMT.  Items of 128 keys, row tiles of up to 64 rows (weigh.cuh).
//
// Items that up to 32 rows see (a decode step): each warp has sixteen keys in
// registers, lanes 2k and 2k + 1 the halves of key k, and goes over the rows, whose dot
// products need one shuffle and whose weights no other thread's.  Bound by the chain of
// loads before the first of them (8 sequences of up to three tokens, 8 heads: 10.7 us; one
// sequence, one token 5.5).
//
// Items of more rows: keys and rows of a tile in shared memory as fp32; thread (ty, tx) of
// 16 x 16 forms the scores of its four rows with the keys tx + 16 j and adds their
// exponentials to the keys' sums, which sixteen threads join at the item's end (three, two or
// one row a thread where a tile has no more).  Two CTAs an SM, so that one's products run
// beside the other's loads (12 single tokens of 28 heads over 12010 rows: 53.7 us, 19
// TFLOP/s, 78.8 with one; bound by the reads of shared memory).

#include <math.h>

#include <atomic>

#include "decode_ptx.cuh"
#include "weigh.cuh"

namespace ecokv {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64;     // rows a row tile
constexpr int kPad = kD + 4;  // floats a padded row: 16-byte reads of 8 consecutive rows meet all banks
constexpr int kFew = 32;      // rows of an item whose keys are split between the warps
constexpr int kOwn = kKeys / (kThreads / 32);  // keys that a warp has

struct Smem {
  float q[kRows][kPad];
  float k[kKeys][kPad];
  float ref[kRows];
  float sum[16][kKeys];
  WeighItem item;
  int more;
};
static_assert(2 * (sizeof(Smem) + 1024) <= 233472, "two CTAs' shared memory");

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xffff0000u));
}

// Offset of key j of the item's source in K, negative: none (a page number out of range).
__device__ __forceinline__ int64_t key_offset(const AttendArgs& a, const WeighItem& it, int j) {
  if (it.source == 0)
    return (a.prefix.head_off ? 0 : (int64_t)it.head * a.prefix.head_stride) +
           ((int64_t)it.row0 + j) * a.prefix.row_stride;
  const int page = a.cache.table[(int64_t)it.seq * a.cache.table_stride + (j >> a.page_shift)];
  if (page < 0 || page >= a.cache.n_pages) {
    note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)it.seq);
    return -1;
  }
  return (int64_t)page * a.cache.page_stride + (int64_t)it.head * a.cache.head_stride +
         (int64_t)(j & (a.cache.page_size - 1)) * a.cache.slot_stride;
}

// Rows r of row tile t: token t * tpt + r / g of the item, its query head r % g.
template <typename T>
__device__ __forceinline__ void load_rows(const WeighArgs& w, Smem& s, const WeighItem& it, int t, int rows) {
  const AttendArgs& a = w.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k0 = t * w.tpt[it.source];
#pragma unroll 4
  for (int r = warp; r < rows; r += kThreads / 32) {
    const int k = r / a.g, token = it.tok0 + k0 + k, hq = it.head * a.g + r - k * a.g;
    *reinterpret_cast<float4*>(&s.q[r][lane * 4]) =
        load4(static_cast<const T*>(a.q) + (int64_t)token * a.q_token + (int64_t)hq * a.q_head + lane * 4);
    if (lane == 0) s.ref[r] = weigh_ref(w.lse[(int64_t)token * a.h_q + hq]);
  }
}

// A key's sum to its weight, or to where the joining kernel finds it.
__device__ __forceinline__ void put(const WeighArgs& w, const WeighItem& it, int k, float sum) {
  if (it.tile0 != 0) {
    w.next[(int64_t)blockIdx.x * kWeighSpan + k] = sum;
    return;
  }
  const int j = it.key0 + k;
  float* at = weight_at(w, it, j);
  if (at != nullptr) *at = weight_after(w, weight_before(it, at, j), sum);
}

template <typename T>
__device__ __forceinline__ void item_few(const WeighArgs& w, Smem& s, const WeighItem& it) {
  const AttendArgs& a = w.a;
  const int lane = threadIdx.x & 31, kk = lane >> 1, half = lane & 1;
  const int k = (threadIdx.x >> 5) * kOwn + kk, j = it.key0 + k, rows = it.ntok * a.g;
  const int64_t at = k < it.nkeys ? key_offset(a, it, j) : -1;
  const T* K = static_cast<const T*>(it.source == 0 ? a.prefix.k : a.cache.k);
  float4 kr[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {  // (every other 16 bytes of the row, its neighbour lane the others)
    kr[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at >= 0) kr[i] = load4(K + at + (2 * i + half) * 4);
  }
  load_rows<T>(w, s, it, 0, rows);
  __syncthreads();
  float sum = 0.f;
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
    const bool seen = it.source == 0 || j <= it.base + r / a.g;
    if (seen) sum += ptx::ex2(fmaf(e, a.scale_log2, s.ref[r]));
  }
  if (half == 0 && k < it.nkeys) put(w, it, k, sum);
}

// The exponentials of a row tile's scores, added over its rows by sixteenth: R rows a thread and
// C keys (16 C of the tile; those that are not there are zeros).  A step's loads come ahead of
// its products: between them they took three times as long.
template <int R, int C>
__device__ __forceinline__ void add_rows(const WeighArgs& w, const Smem& s, const WeighItem& it, int t, int rows,
                                         float (&total)[8]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float x[R][C];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c) x[r][c] = 0.f;
#pragma unroll 1
  for (int e = 0; e < kD; e += 4) {
    float4 q4[R], k4[C];
#pragma unroll
    for (int r = 0; r < R; ++r) q4[r] = *reinterpret_cast<const float4*>(&s.q[ty * R + r][e]);
#pragma unroll
    for (int c = 0; c < C; ++c) k4[c] = *reinterpret_cast<const float4*>(&s.k[tx + 16 * c][e]);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        x[r][c] = fmaf(q4[r].x, k4[c].x, x[r][c]);
        x[r][c] = fmaf(q4[r].y, k4[c].y, x[r][c]);
        x[r][c] = fmaf(q4[r].z, k4[c].z, x[r][c]);
        x[r][c] = fmaf(q4[r].w, k4[c].w, x[r][c]);
      }
  }
  float sum[C];
#pragma unroll
  for (int c = 0; c < C; ++c) sum[c] = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = ty * R + r;
    if (row < rows) {  // (what shared memory holds past them may be anything)
      const float ref = s.ref[row];
      const int seen = it.source == 0 ? it.nkeys : it.base + t * w.tpt[1] + row / w.a.g + 1 - it.key0;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (tx + 16 * c < seen) sum[c] += ptx::ex2(fmaf(x[r][c], w.a.scale_log2, ref));
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) total[c] += sum[c];
}
template <int R>
__device__ __forceinline__ void add_rows(const WeighArgs& w, const Smem& s, const WeighItem& it, int t, int rows,
                                         float (&total)[8]) {
  if (it.nkeys > 64) add_rows<R, 8>(w, s, it, t, rows, total);
  else if (it.nkeys > 16) add_rows<R, 4>(w, s, it, t, rows, total);
  else add_rows<R, 1>(w, s, it, t, rows, total);
}

template <typename T>
__device__ __forceinline__ void item_rows(const WeighArgs& w, Smem& s, const WeighItem& it) {
  const AttendArgs& a = w.a;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 31, warp = tid >> 5;
  const T* K = static_cast<const T*>(it.source == 0 ? a.prefix.k : a.cache.k);
  const int tpt = w.tpt[it.source];
  {
    // offsets, in the place of the sums
    int64_t* at = reinterpret_cast<int64_t*>(&s.sum[0][0]);
    if (tid < kKeys) at[tid] = tid < it.nkeys ? key_offset(a, it, it.key0 + tid) : -1;
    __syncthreads();
#pragma unroll 8
    for (int i = 0; i < kKeys / (kThreads / 32); ++i) {
      const int kk = warp + i * (kThreads / 32);
      float4 k4 = make_float4(0.f, 0.f, 0.f, 0.f);
      if (at[kk] >= 0) k4 = load4(K + at[kk] + lane * 4);
      *reinterpret_cast<float4*>(&s.k[kk][lane * 4]) = k4;
    }
  }
  float total[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) total[c] = 0.f;
#pragma unroll 1
  for (int t = it.tile0; t < it.tile0 + it.ntiles; ++t) {
    const int rows = min(it.ntok - t * tpt, tpt) * a.g;
    __syncthreads();
    load_rows<T>(w, s, it, t, rows);
    __syncthreads();
    if (rows <= 16) add_rows<1>(w, s, it, t, rows, total);
    else if (rows <= 32) add_rows<2>(w, s, it, t, rows, total);
    else if (rows <= 48) add_rows<3>(w, s, it, t, rows, total);
    else add_rows<4>(w, s, it, t, rows, total);
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < 8; ++c) s.sum[ty][tx + 16 * c] = total[c];
  __syncthreads();
  if (tid < it.nkeys) {
    float sum = 0.f;
#pragma unroll
    for (int y = 0; y < 16; ++y) sum += s.sum[y][tid];
    put(w, it, tid, sum);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) weigh_simt_kernel(const __grid_constant__ WeighArgs w) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Smem& s = *reinterpret_cast<Smem*>(smem_raw);
  const int lane = threadIdx.x & 31;
  ptx::grid_wait();
  WeighWalk walk;
  bool first = true;
  if (threadIdx.x < 32) walk.begin(w, blockIdx.x, lane, blockIdx.x == 0);
  while (true) {
    __syncthreads();
    if (threadIdx.x < 32) {
      WeighItem it{};
      const bool more = walk.next(w, it);
      if (lane == 0) {
        s.item = it;
        s.more = more ? 1 : 0;
        if (first) w.next_item[blockIdx.x] = it;
      }
      first = false;
    }
    __syncthreads();
    if (s.more == 0) break;
    const WeighItem it = s.item;
    if (it.ntok <= w.tpt[it.source] && it.ntok * w.a.g <= kFew) item_few<T>(w, s, it);
    else item_rows<T>(w, s, it);
  }
  ptx::grid_trigger();
}

template <typename T>
cudaError_t launch(const WeighArgs& w, cudaStream_t st) {
  static std::atomic<bool> set[64];  // a racing thread repeats the idempotent setting
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!set[dev].load()) {
    e = cudaFuncSetAttribute(weigh_simt_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
    if (e != cudaSuccess) return e;
    set[dev].store(true);
  }
  return launch_behind(weigh_simt_kernel<T>, (unsigned)w.a.P, kThreads, sizeof(Smem), st, w);
}

}  // namespace

cudaError_t launch_weigh_simt(const WeighArgs& w, ecokv_dtype dt, cudaStream_t st) {
  return dt == ECOKV_F32 ? launch<float>(w, st) : launch<__nv_bfloat16>(w, st);
}

}  // namespace ecokv
