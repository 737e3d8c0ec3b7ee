// ecokv_prune: the slots that stay, by weight, and the move of their rows.  A cluster has a
// (sequence, head): half of its CTAs move the rows of K and half those of V.  While all
// clusters are resident at once, the first CTA of each chooses the slots before that (40 heads
// of up to 1500 slots: 11.5 us, 13.8 in two kernels); otherwise a kernel before it does,
// so that no CTA waits in the place of one that moves (256 heads of up to 4097 slots: 43.8 us,
// 63.9 in one; the choice is latency, 10 us, the move 33, 180 MB at 5.4 TB/s).

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

// The slots of (sequence b, head h) that stay, L being more than the limit, by one CTA.  The need-th largest key of the slots between the fixed ones is
// found digit by digit (11, 11 and 10 bits) in histograms; the slots above it stay, and
// the lowest of those that equal it.  A warp has a run of 32's of slots, so that
// their places follow from counts of the warps before it.  Keys are read from memory once
// (those past the shared memory four times).
constexpr int kThreads = 512;  // of a CTA that chooses
constexpr int kWarps = kThreads / 32;
constexpr int kMoveThreads = 256;  // of one that only moves: all of 256 heads' are resident
constexpr int kBins = 2048;
constexpr int kAhead = 8;

struct SelectSmem {
  unsigned bins[kBins];
  unsigned part[kWarps];
  unsigned found[3];
  int2 count[kWarps];
};

__device__ __forceinline__ void select_slots(const PruneArgs& a, SelectSmem& s, unsigned* keys, int b, int h, int L,
                                             int32_t* out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = a.budget + tid; i < a.limit; i += kThreads) out[i] = -1;
  for (int i = tid; i < a.first; i += kThreads) out[i] = i;
  for (int i = tid; i < a.recent; i += kThreads) out[a.budget - a.recent + i] = L - a.recent + i;
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
    for (int i = tid; i < kBins; i += kThreads) s.bins[i] = 0;
    __syncthreads();
    if (pass == 0) {
#pragma unroll 1
      for (int i0 = tid; i0 < n; i0 += kAhead * kThreads) {  // (as many loads at once)
        int page[kAhead];
        float x[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) page[j] = page_of(min(i0 + j * kThreads, n - 1));
#pragma unroll
        for (int j = 0; j < kAhead; ++j) x[j] = load(min(i0 + j * kThreads, n - 1), page[j]);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int i = i0 + j * kThreads;
          if (i >= n) break;
          if (page[j] < 0 || page[j] >= a.m.from.n_pages) flag(a.m.status, (unsigned)b);
          const unsigned k = order_of(x[j]);
          if (i < a.cached) keys[i] = k;
          atomicAdd(&s.bins[k >> 21], 1u);
        }
      }
    } else {
#pragma unroll 4
      for (int i = tid; i < n; i += kThreads) {
        const unsigned k = key(i);
        if (((k ^ top) >> (low + width)) == 0) atomicAdd(&s.bins[(k >> low) & ((1u << width) - 1)], 1u);
      }
    }
    __syncthreads();
    // from the top bin down: the one in which the count reaches `left`
    constexpr int kPer = kBins / kThreads;
    unsigned mine[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      mine[j] = s.bins[kBins - 1 - (tid * kPer + j)];
      sum += mine[j];
    }
    unsigned upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned u = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += u;
    }
    if (lane == 31) s.part[warp] = upto;
    __syncthreads();
    unsigned before = upto - sum;
    for (int w = 0; w < warp; ++w) before += s.part[w];
    if (before < left && before + sum >= left) {  // (one thread)
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        if (before < left && before + mine[j] >= left) {
          s.found[0] = (unsigned)(kBins - 1 - (tid * kPer + j));
          s.found[1] = left - before;
          s.found[2] = mine[j];
        }
        before += mine[j];
      }
    }
    __syncthreads();
    top |= s.found[0] << low;
    left = s.found[1];
    if (s.found[2] == left) {  // all of the digits so far stay: those above the next lower key
      left = 0;
      top -= 1;  // (0: NaN alone, of which never all stay)
      break;
    }
  }
  const int equal = (int)left;  // slots of the key `top` that stay, the lowest ones
  const int run = (div_up(n, kThreads)) * 32, i0 = warp * run, i1 = min(i0 + run, n);
  int gt = 0, eq = 0;
  for (int i = i0; i < i1; i += 32) {
    const unsigned k = i + lane < i1 ? key(i + lane) : 0u;
    gt += __popc(__ballot_sync(0xffffffffu, i + lane < i1 && k > top));
    eq += __popc(__ballot_sync(0xffffffffu, i + lane < i1 && k == top));
  }
  if (lane == 0) s.count[warp] = make_int2(gt, eq);
  __syncthreads();
  gt = eq = 0;
  for (int w = 0; w < warp; ++w) {
    gt += s.count[w].x;
    eq += s.count[w].y;
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

__device__ __forceinline__ void choose(const PruneArgs& a, SelectSmem& s, unsigned* keys, int b, int h, int L,
                                       int32_t* list) {
  if (L > a.limit) {
    select_slots(a, s, keys, b, h, L, list);
  } else {
    for (int i = threadIdx.x; i < a.limit; i += kThreads) list[i] = i < L ? i : -1;
  }
}

__global__ void __launch_bounds__(kThreads) prune_select_kernel(const __grid_constant__ PruneArgs a) {
  extern __shared__ unsigned keys[];
  __shared__ SelectSmem select;
  ptx::grid_trigger();
  ptx::grid_wait();
  const int b = blockIdx.x / a.m.h_kv, h = blockIdx.x - b * a.m.h_kv;
  const int L = length_of(a, b, threadIdx.x == 0 && h == 0 ? a.m.status : nullptr);
  choose(a, select, keys, b, h, L, a.idx + (int64_t)blockIdx.x * a.limit);
}

template <int E, bool kChoose>
__global__ void __launch_bounds__(kChoose ? kThreads : kMoveThreads, kChoose ? 2 : 4)
    prune_move_kernel(const __grid_constant__ PruneArgs a) {
  extern __shared__ unsigned keys[];
  ptx::grid_trigger();
  ptx::grid_wait();
  const int per = 2 * a.m.ctas, unit = blockIdx.x / per, rank = blockIdx.x - unit * per, kv = rank & 1;
  const int b = unit / a.m.h_kv, h = unit - b * a.m.h_kv;
  const bool lead = rank == 0 && h == 0;
  const int L = length_of(a, b, kChoose && lead && threadIdx.x == 0 ? a.m.status : nullptr);
  const bool cut = L > a.limit;
  const int n = cut ? a.budget : L;
  int32_t* list = a.idx + (int64_t)unit * a.limit;
  if constexpr (kChoose) {
    __shared__ SelectSmem select;
    if (rank == 0) choose(a, select, keys, b, h, L, list);
  }
  if (a.lengths_out != nullptr && lead && threadIdx.x == 0) a.lengths_out[b] = n;
  // (in the same cache the first ones stay where they are, and so does a sequence that is not cut)
  const int i0 = a.m.in_place ? (cut ? a.first : n) : 0;
  if (i0 >= n) return;
  if (kChoose && cut) cooperative_groups::this_cluster().sync();  // the list is there
  move_rows<E, kChoose ? kThreads : kMoveThreads>(a.m, b, h, kv, rank >> 1, i0, n, 0, [=](int i) { return cut ? list[i] : i; });
}

// The lengths alone, once nothing reads the old ones any more.
__global__ void __launch_bounds__(kThreads) prune_lengths_kernel(const __grid_constant__ PruneArgs a) {
  ptx::grid_trigger();
  ptx::grid_wait();
  const int b = blockIdx.x * kThreads + threadIdx.x;
  if (b >= a.m.batch) return;
  const int L = length_of(a, b, nullptr);
  a.lengths_out[b] = L > a.limit ? a.budget : L;
}

constexpr int kMostCached = 16 * 1024;  // slots

cudaError_t launch(const PruneArgs& a, ecokv_dtype dt, int64_t units, bool choose, cudaStream_t st) {
  auto move = choose ? (dt == ECOKV_F32 ? prune_move_kernel<4, true> : prune_move_kernel<2, true>)
                     : (dt == ECOKV_F32 ? prune_move_kernel<4, false> : prune_move_kernel<2, false>);
  static std::atomic<bool> set[64];  // a racing thread repeats the idempotent setting
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!set[dev].load()) {
    for (auto* k : {prune_move_kernel<4, true>, prune_move_kernel<2, true>, prune_select_kernel})
      if ((e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostCached * 4)) != cudaSuccess)
        return e;
    set[dev].store(true);
  }
  const size_t smem = (size_t)a.cached * 4;
  if (!choose && (e = launch_behind(prune_select_kernel, (unsigned)units, kThreads, smem, st, a)) != cudaSuccess)
    return e;
  return launch_move(move, a.m, (unsigned)(units * 2 * a.m.ctas), choose ? kThreads : kMoveThreads, choose ? smem : 0,
                     st, a);
}

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
  // (in the same cache rows that stay in place are not touched, nor are their weights)
  if (to == nullptr && to_weights != nullptr &&
      (to_weights->w != weights->w || to_weights->page_stride != weights->page_stride ||
       to_weights->head_stride != weights->head_stride || to_weights->slot_stride != weights->slot_stride))
    return ECOKV_ERR_INVALID_ARG;
  if ((int64_t)p->batch * p->h_kv > 1 << 29) return ECOKV_ERR_UNSUPPORTED;
  if (!idx || ((uintptr_t)idx & 3u) || !lengths_ok(cache->lengths, lengths_out, p->batch) ||
      !apart(idx, (int64_t)p->batch * p->h_kv * p->limit, lengths_out, p->batch) ||
      !apart(idx, (int64_t)p->batch * p->h_kv * p->limit, cache->lengths, p->batch))
    return ECOKV_ERR_INVALID_ARG;
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
  const int64_t units = (int64_t)p->batch * p->h_kv, rows = to != nullptr ? p->limit : p->budget;
  // two CTAs a unit, and more while all of them together are no more than two an SM and have a chunk
  // each, up to a cluster's eight
  const int64_t sms = attend_sms();
  const int64_t chunk = kMoveBytes / (kD * (dtype == ECOKV_F32 ? 4 : 2));
  a.m.ctas = 1;
  while (a.m.ctas < 4 && units * 2 * a.m.ctas < sms && chunk * a.m.ctas < rows) a.m.ctas *= 2;
  const bool choose = units * 2 * a.m.ctas <= 2 * sms;
  a.m.cluster = choose ? 2 * a.m.ctas : 1;
  const bool same = lengths_out == cache->lengths;
  a.lengths_out = same ? nullptr : lengths_out;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = launch(a, dtype, units, choose, s);
  if (e == cudaSuccess && same) {
    a.lengths_out = lengths_out;
    e = launch_behind(prune_lengths_kernel, (unsigned)div_up(p->batch, kThreads), kThreads, 0, s, a);
  }
  return e == cudaSuccess ? ECOKV_OK : ECOKV_ERR_CUDA;
}
