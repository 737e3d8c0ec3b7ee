// ecokv_prune: the slots that stay, by weight, and the move of their rows.

#include <atomic>

#include "cache_move.cuh"

namespace ecokv {
namespace {

struct PruneArgs {
  MoveArgs m;
  ecokv_weights w;
  int32_t* idx;
  int32_t* lengths_out;  // NULL: another kernel's
  int budget, limit, first, recent, cap;
  int cached;            // slots whose keys are kept in shared memory
};

__device__ __forceinline__ int length_of(const PruneArgs& a, int b, unsigned* status) {
  const int len = a.m.from.lengths[b], L = min(max(len, 0), a.cap);
  if (L != len) flag(status, (unsigned)b);
  return L;
}

// A number in an unsigned order: -0 as 0, NaN below all.
__device__ __forceinline__ unsigned order_of(float x) {
  if (x != x) return 0u;
  const unsigned u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// One CTA a (sequence, head).  The need-th largest key of the slots between the fixed ones is
// found digit by digit (11, 11 and 10 bits) in histograms; the slots above it stay, and
// the lowest of those that equal it.  A warp has a run of 32's of slots, so that
// their places follow from counts of the warps before it.  Keys are read from memory once
// (those past the shared memory four times).
constexpr int kSelectThreads = 512;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kBins = 2048;
constexpr int kAhead = 8;

__global__ void __launch_bounds__(kSelectThreads) prune_select_kernel(const __grid_constant__ PruneArgs a) {
  extern __shared__ unsigned keys[];
  __shared__ unsigned bins[kBins];
  __shared__ unsigned part[kSelectWarps];
  __shared__ unsigned found[2];
  __shared__ int2 count[kSelectWarps];
  ptx::grid_trigger();
  ptx::grid_wait();
  const int b = blockIdx.x / a.m.h_kv, h = blockIdx.x - b * a.m.h_kv;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int32_t* out = a.idx + (int64_t)blockIdx.x * a.limit;
  const int L = length_of(a, b, tid == 0 && h == 0 ? a.m.status : nullptr);
  if (L <= a.limit) {
    for (int i = tid; i < a.limit; i += kSelectThreads) out[i] = i < L ? i : -1;
    return;
  }
  for (int i = a.budget + tid; i < a.limit; i += kSelectThreads) out[i] = -1;
  for (int i = tid; i < a.first; i += kSelectThreads) out[i] = i;
  for (int i = tid; i < a.recent; i += kSelectThreads) out[a.budget - a.recent + i] = L - a.recent + i;
  const int need = a.budget - a.first - a.recent, n = L - a.first - a.recent;  // need < n
  if (need == 0) return;
  const int* table = a.m.from.table + (int64_t)b * a.m.from.table_stride;
  const float* weights = a.w.w + (int64_t)h * a.w.head_stride;
  auto page_of = [&](int i) { return table[(a.first + i) >> a.m.from_shift]; };
  auto load = [&](int i, int page) {
    const int row = (a.first + i) & (a.m.from.page_size - 1);
    return page < 0 || page >= a.m.from.n_pages
               ? -INFINITY
               : weights[(int64_t)page * a.w.page_stride + (int64_t)row * a.w.slot_stride];
  };
  auto key = [&](int i) { return i < a.cached ? keys[i] : order_of(load(i, page_of(i))); };

  unsigned top = 0;       // the key's digits so far
  unsigned left = need;   // keys of these digits that stay
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0;   // bits below the digit
    const int width = pass == 2 ? 10 : 11;
    for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    if (pass == 0) {
#pragma unroll 1
      for (int i0 = tid; i0 < n; i0 += kAhead * kSelectThreads) {  // (as many loads at once)
        int page[kAhead];
        float x[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) page[j] = page_of(min(i0 + j * kSelectThreads, n - 1));
#pragma unroll
        for (int j = 0; j < kAhead; ++j) x[j] = load(min(i0 + j * kSelectThreads, n - 1), page[j]);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int i = i0 + j * kSelectThreads;
          if (i >= n) break;
          if (page[j] < 0 || page[j] >= a.m.from.n_pages) flag(a.m.status, (unsigned)b);
          const unsigned k = order_of(x[j]);
          if (i < a.cached) keys[i] = k;
          atomicAdd(&bins[k >> 21], 1u);
        }
      }
    } else {
#pragma unroll 4
      for (int i = tid; i < n; i += kSelectThreads) {
        const unsigned k = key(i);
        if (((k ^ top) >> (low + width)) == 0) atomicAdd(&bins[(k >> low) & ((1u << width) - 1)], 1u);
      }
    }
    __syncthreads();
    // from the top bin down: the one in which the count reaches `left`
    constexpr int kPer = kBins / kSelectThreads;
    unsigned mine[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      mine[j] = bins[kBins - 1 - (tid * kPer + j)];
      sum += mine[j];
    }
    unsigned upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned u = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += u;
    }
    if (lane == 31) part[warp] = upto;
    __syncthreads();
    unsigned before = upto - sum;
    for (int w = 0; w < warp; ++w) before += part[w];
    if (before < left && before + sum >= left) {  // (one thread)
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        if (before < left && before + mine[j] >= left) {
          found[0] = (unsigned)(kBins - 1 - (tid * kPer + j));
          found[1] = left - before;
        }
        before += mine[j];
      }
    }
    __syncthreads();
    top |= found[0] << low;
    left = found[1];
  }
  const int equal = (int)left;  // slots of the key `top` that stay, the lowest ones
  const int run = (div_up(n, kSelectThreads)) * 32, i0 = warp * run, i1 = min(i0 + run, n);
  int gt = 0, eq = 0;
  for (int i = i0; i < i1; i += 32) {
    const unsigned k = i + lane < i1 ? key(i + lane) : 0u;
    gt += __popc(__ballot_sync(0xffffffffu, i + lane < i1 && k > top));
    eq += __popc(__ballot_sync(0xffffffffu, i + lane < i1 && k == top));
  }
  if (lane == 0) count[warp] = make_int2(gt, eq);
  __syncthreads();
  gt = eq = 0;
  for (int w = 0; w < warp; ++w) {
    gt += count[w].x;
    eq += count[w].y;
  }
  const unsigned below = (1u << lane) - 1;
  for (int i = i0; i < i1; i += 32) {
    const unsigned k = i + lane < i1 ? key(i + lane) : 0u;
    const bool is_gt = i + lane < i1 && k > top, is_eq = i + lane < i1 && k == top;
    const unsigned mg = __ballot_sync(0xffffffffu, is_gt), me = __ballot_sync(0xffffffffu, is_eq);
    const int e = eq + __popc(me & below);
    if (is_gt || (is_eq && e < equal))
      out[a.first + gt + __popc(mg & below) + min(e, equal)] = a.first + i + lane;
    gt += __popc(mg);
    eq += __popc(me);
  }
}

template <int E>
__global__ void __launch_bounds__(kMoveThreads, 4) prune_move_kernel(const __grid_constant__ PruneArgs a) {
  ptx::grid_trigger();
  ptx::grid_wait();
  const int unit = blockIdx.x / a.m.ctas, rank = blockIdx.x - unit * a.m.ctas;
  const int kv = unit & 1, h = (unit >> 1) % a.m.h_kv, b = (unit >> 1) / a.m.h_kv;
  const int L = length_of(a, b, nullptr);
  const bool cut = L > a.limit;
  const int n = cut ? a.budget : L;
  const int32_t* list = a.idx + ((int64_t)b * a.m.h_kv + h) * a.limit;
  // (in the same cache the first ones stay where they are, and so does a sequence that is not cut)
  const int i0 = a.m.in_place ? (cut ? a.first : n) : 0;
  move_rows<E>(a.m, b, h, kv, rank, i0, n, 0, [=](int i) { return list[i]; });
  if (a.lengths_out != nullptr && h == 0 && kv == 0 && rank == 0 && threadIdx.x == 0) a.lengths_out[b] = n;
}

// The lengths alone, once nothing reads the old ones any more.
__global__ void __launch_bounds__(kMoveThreads) prune_lengths_kernel(const __grid_constant__ PruneArgs a) {
  ptx::grid_trigger();
  ptx::grid_wait();
  const int b = blockIdx.x * kMoveThreads + threadIdx.x;
  if (b >= a.m.batch) return;
  const int L = length_of(a, b, nullptr);
  a.lengths_out[b] = L > a.limit ? a.budget : L;
}

constexpr int kMostCached = 48 * 1024;  // slots

}  // namespace
}  // namespace ecokv

using namespace ecokv;

extern "C" ecokv_status ecokv_prune(const ecokv_prune_params* p, ecokv_dtype dtype, const ecokv_pages* cache,
                                    const ecokv_weights* weights, const ecokv_pages* to,
                                    const ecokv_weights* to_weights, int32_t* idx, int32_t* lengths_out, void* ws,
                                    size_t ws_bytes, void* stream) {
  if (p == nullptr || (dtype != ECOKV_F32 && dtype != ECOKV_BF16)) return ECOKV_ERR_INVALID_ARG;
  if (p->h_kv < 1 || p->batch < 1 || p->first < 0 || p->recent < 0 || p->budget < 1 || p->limit < p->budget ||
      (int64_t)p->first + p->recent > p->budget)
    return ECOKV_ERR_INVALID_ARG;
  ecokv_status st = check_pages(cache, p->batch, dtype);
  if (st == ECOKV_OK && to != nullptr) {
    ecokv_pages c = *to;
    c.lengths = cache->lengths;  // (not read)
    st = check_pages(&c, p->batch, dtype);
  }
  if (st != ECOKV_OK) return st;
  if (weights == nullptr || !weights_ok(weights) || (to_weights != nullptr && !weights_ok(to_weights)))
    return ECOKV_ERR_INVALID_ARG;
  if (!idx || ((uintptr_t)idx & 3u) || !lengths_ok(cache->lengths, lengths_out, p->batch)) return ECOKV_ERR_INVALID_ARG;
  if ((int64_t)p->batch * p->h_kv > 1 << 29) return ECOKV_ERR_UNSUPPORTED;
  if (ws != nullptr && (!aligned16(ws) || ws_bytes < 256)) return ECOKV_ERR_WORKSPACE;
  PruneArgs a{};
  a.m.from = *cache;
  a.m.to = to != nullptr ? *to : *cache;
  a.m.from_shift = __builtin_ctz((unsigned)a.m.from.page_size);
  a.m.to_shift = __builtin_ctz((unsigned)a.m.to.page_size);
  a.w = *weights;
  if (to_weights != nullptr) {
    a.m.w_from = *weights;
    a.m.w_to = *to_weights;
  }
  a.m.h_kv = p->h_kv;
  a.m.batch = p->batch;
  a.m.in_place = to == nullptr;
  a.m.status = static_cast<unsigned*>(ws);
  a.idx = idx;
  a.budget = p->budget;
  a.limit = p->limit;
  a.first = p->first;
  a.recent = p->recent;
  a.cap = cache->page_size * cache->table_stride;
  a.cached = a.cap < kMostCached ? a.cap : kMostCached;
  a.m.ctas = move_ctas(2ll * p->batch * p->h_kv, to != nullptr ? p->limit : p->budget, dtype);
  const bool same = lengths_out == cache->lengths;
  a.lengths_out = same ? nullptr : lengths_out;
  static std::atomic<bool> set[64];  // a racing thread repeats the idempotent setting
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return ECOKV_ERR_CUDA;
  if (!set[dev].load()) {
    if (cudaFuncSetAttribute(prune_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostCached * 4) !=
        cudaSuccess)
      return ECOKV_ERR_CUDA;
    set[dev].store(true);
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = launch_behind(prune_select_kernel, (unsigned)(p->batch * p->h_kv), kSelectThreads,
                                (size_t)a.cached * 4, s, a);
  if (e == cudaSuccess)
    e = dtype == ECOKV_F32 ? launch_move(prune_move_kernel<4>, a.m, s, a) : launch_move(prune_move_kernel<2>, a.m, s, a);
  if (e == cudaSuccess && same) {
    a.lengths_out = lengths_out;
    e = launch_behind(prune_lengths_kernel, (unsigned)div_up(p->batch, kMoveThreads), kMoveThreads, 0, s, a);
  }
  return e == cudaSuccess ? ECOKV_OK : ECOKV_ERR_CUDA;
}
