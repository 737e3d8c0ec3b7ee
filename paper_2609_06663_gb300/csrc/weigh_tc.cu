// Weights of keys on the tensor cores (bf16): items and row tiles as in weigh.cuh, one
// persistent CTA an SM.
//
// S^T = K Q^T: a key tile is the M of the product, a row tile its N (as many columns as it
// has rows, in sixteens), so that a thread has a key: it adds the exponentials of its
// row of S^T, whose references lie in shared memory, in registers, without a shuffle and
// without a maximum, the sums of exponentials being known.  An item's two key tiles stay in
// shared memory while the row tiles pass by; each has two accumulators in tensor memory, for
// even and odd row tiles of all items, and each accumulator a warpgroup ("stream") of its
// own, so that the products run beside the exponentials and four warps a scheduler hide
// each other's latencies.  The sums of an item's even and odd tiles are added at its end.
//
// Bound by the keys' bytes where few rows see them (64 sequences of up to 4097 slots and a
// token each, 28 heads over 4: 31.0 us, 4.9 TB/s over the call, of which 8 are the walk's
// start and the launch).  Where many do (806 tokens over 6554 rows: 45.5 us, 841 TFLOP/s) a
// stream takes 5100 cycles a row tile: 3240 for its 128 columns, 380 waiting for their
// references, 260 for the product, 120 for the other stream's sum.  A CTA's four
// streams share a unit for exponentials that 2048 would do and a tensor pipe that 2200
// would: without exponentials it takes 44 us, with half of each product 45, with half of
// the columns 36.
//
// Warps: 0 copies (TMA; a lane a page), 1 the products, 2 the walk over the items, 3 the
// rows' references, 4-19 the streams: key tile, then parity.

#include <atomic>

#include "decode_ptx.cuh"
#include "tc_tile.cuh"
#include "weigh.cuh"

namespace ecokv {
namespace {

using namespace ptx;

constexpr int kThreads = 640;
constexpr int kKeyTiles = 4;  // key tiles in the ring
constexpr int kRowTiles = 3;  // row tiles (two: 53.7 us for 806 tokens over 6554 rows, three 46.9)
constexpr int kRefs = 2;      // row tiles' references, one of each parity
constexpr int kItems = 4;     // items ahead of their consumers
constexpr uint32_t kHalf = kTileBytes / 2;  // 128 rows x 64 columns

struct Smem {
  uint8_t k[kKeyTiles][kTileBytes];
  uint8_t q[kRowTiles][kTileBytes];
  float ref[kRefs][128];
  uint64_t kfull[kKeyTiles], kempty[kKeyTiles];
  uint64_t qfull[kRowTiles], qempty[kRowTiles], rfull[kRefs], rempty[kRefs];
  uint64_t sfull[2][2], sempty[2][2];  // [key tile][parity]
  uint64_t mready[2][4], mdone[2][4];  // between the streams' warps of the same keys
  float sum[2][128];                   // of the stream that has not had the item's first tile
  uint64_t ifull[kItems], iempty[kItems];
  uint64_t drained;
  WeighItem items[kItems];
  uint32_t tmem;
  volatile int abort;
};
static_assert(sizeof(Smem) <= 232448, "one CTA's shared memory");

struct Maps {
  CUtensorMap q[2], pk, ck;
};

// Bounded wait: false once this CTA has given up (the clock is read every 16th try).
__device__ __noinline__ bool wait_long(Smem& s, const AttendArgs& a, uint64_t* bar, uint32_t parity, unsigned where) {
  unsigned long long t0 = 0;
#pragma unroll 1
  for (uint32_t i = 1; !mbar_try_wait(bar, parity); ++i) {
    if ((i & 15u) != 0) continue;
    if (s.abort) return false;
    const unsigned long long t = now_ns();
    if (t0 == 0) t0 = t;
    if (t - t0 > a.timeout_ns) {
      s.abort = 1;
      note(a, ECOKV_ERR_TIMEOUT, where);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool wait_bar(Smem& s, const AttendArgs& a, uint64_t* bar, uint32_t parity, unsigned where) {
  return mbar_try_wait(bar, parity) || wait_long(s, a, bar, parity, where);
}
// A whole warp's wait.
__device__ __forceinline__ bool wait_warp(Smem& s, const AttendArgs& a, uint64_t* bar, uint32_t parity,
                                          unsigned where) {
  return __all_sync(0xffffffffu, wait_bar(s, a, bar, parity, where)) != 0;
}

// A place in a ring of n and the parity of its phase.
template <int n>
struct Ring {
  uint32_t at = 0, phase = 0;
  __device__ __forceinline__ void step() {
    if (++at == n) {
      at = 0;
      phase ^= 1;
    }
  }
};

// The next item of the queue, for a warp; false: none left, or given up.
struct ItemReader {
  Ring<kItems> r;
  __device__ __forceinline__ bool next(Smem& s, const AttendArgs& a, WeighItem& it, int lane) {
    if (!wait_warp(s, a, &s.ifull[r.at], r.phase, 1u)) return false;
    it = s.items[r.at];
    __syncwarp();
    if (lane == 0) mbar_arrive(&s.iempty[r.at]);
    r.step();
    return it.ntiles > 0;
  }
};

__device__ __forceinline__ int key_tiles(const WeighItem& it) { return it.nkeys > kKeys ? 2 : 1; }
// Rows of row tile t.
__device__ __forceinline__ int rows_of(const WeighArgs& w, const WeighItem& it, int t) {
  const int tpt = w.tpt[it.source];
  return max(min(it.ntok - t * tpt, tpt), 0) * w.a.g;
}

// What has been issued, for those who wait for it to land.
struct Issued {
  uint32_t k = 0, q = 0;
};

__device__ __forceinline__ void produce(Smem& s, const WeighArgs& w, const Maps& m, int lane, Issued& d) {
  const AttendArgs& a = w.a;
  ItemReader items;
  WeighItem next{};
  Ring<kKeyTiles> kr;
  Ring<kRowTiles> qr;
  int pages[2] = {0, 0};  // this lane's of the next item's key tiles
  auto look_up = [&]() {
    if (next.source == 0) return;
    const int* table = a.cache.table + (int64_t)next.seq * a.cache.table_stride;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int from = next.key0 + p * kKeys, to = min(from + kKeys, next.key0 + next.nkeys);
      const int c = (from >> a.page_shift) + lane;
      if (from < to && c <= (to - 1) >> a.page_shift) pages[p] = table[c];
    }
  };
  bool more = items.next(s, a, next, lane);
  if (more) look_up();
  while (more) {
    const WeighItem it = next;
    const bool own = it.source != 0;
    const int head = own || a.prefix.head_off == nullptr ? it.head : 0;
    const uint32_t box = own ? (uint32_t)min(a.cache.page_size, kKeys) : kKeys;
    const uint32_t at = own ? (((uint32_t)lane << a.page_shift) & (kKeys - 1)) * 128u : lane * kHalf;
    const int nk = key_tiles(it);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      if (p >= nk) break;
      const int from = it.key0 + p * kKeys, to = min(from + kKeys, it.key0 + it.nkeys);
      const int n = own ? ((to - 1) >> a.page_shift) - (from >> a.page_shift) + 1 : 2;
      const int row = own ? from & (a.cache.page_size - 1) : it.row0 + from;
      if (!wait_warp(s, a, &s.kempty[kr.at], kr.phase ^ 1, 2u)) return;
      int page = pages[p];
      if (own && lane < n && (page < 0 || page >= a.cache.n_pages)) {
        note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)it.seq);
        page = a.cache.n_pages;  // out of the map's bounds: zeros
      }
      uint8_t* dst = s.k[kr.at] + at;
      uint64_t* bar = &s.kfull[kr.at];
      if (lane == 0) mbar_expect_tx(bar, own ? box * n * 256u : kTileBytes);
      __syncwarp();
      if (lane < n) {
        if (own) {
          tma_load_4d(dst, &m.ck, bar, 0, row, head, page);
          tma_load_4d(dst + kHalf, &m.ck, bar, 64, row, head, page);
        } else {
          tma_load_3d(dst, &m.pk, bar, lane * 64, row, head);
        }
      }
      kr.step();
      ++d.k;
    }
    // (page numbers an item ahead, on their way while this one's rows are copied)
    more = items.next(s, a, next, lane);
    if (more) look_up();
    const int tpt = w.tpt[it.source];
    for (int t = it.tile0; t < it.tile0 + it.ntiles; ++t) {
      if (!wait_warp(s, a, &s.qempty[qr.at], qr.phase ^ 1, 3u)) return;
      if (lane == 0) mbar_expect_tx(&s.qfull[qr.at], (uint32_t)(tpt * a.g) * 256u);
      __syncwarp();
      if (lane < 2)
        tma_load_3d(s.q[qr.at] + lane * kHalf, &m.q[it.source], &s.qfull[qr.at], lane * 64, it.head * a.g,
                    it.tok0 + t * tpt);
      qr.step();
      ++d.q;
    }
  }
}

// The products, by one thread.
__device__ __forceinline__ void multiply(Smem& s, const WeighArgs& w, uint32_t tmem) {
  const AttendArgs& a = w.a;
  Ring<kItems> ir;
  Ring<kKeyTiles> kr;
  Ring<kRowTiles> qr;
  uint32_t n = 0;         // row tiles so far
  uint32_t phase = 0;     // bit 2 p + b: parity of the next phase of sempty[p][b]
  const uint64_t k0 = smem_desc(smem_u32(s.k[0]), 16, 1024, 2), q0 = smem_desc(smem_u32(s.q[0]), 16, 1024, 2);
  while (true) {
    if (!wait_bar(s, a, &s.ifull[ir.at], ir.phase, 1u)) return;
    const WeighItem it = s.items[ir.at];
    mbar_arrive(&s.iempty[ir.at]);
    ir.step();
    if (it.ntiles <= 0) return;
    const int nk = key_tiles(it);
    uint32_t slot[2] = {0, 0};
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (p < nk) slot[p] = kr.at, kr.step();
    for (int t = it.tile0; t < it.tile0 + it.ntiles; ++t, ++n) {
      const uint32_t cols = (uint32_t)max((rows_of(w, it, t) + 15) & ~15, 16), b = n & 1;
      const uint32_t idesc = idesc_bf16(128, (int)cols, false, false);
      if (!wait_bar(s, a, &s.qfull[qr.at], qr.phase, 4u)) return;
      const uint64_t qd = q0 + (uint64_t)(qr.at * (kTileBytes >> 4));
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (p >= nk) break;
        if (t == it.tile0) {
          // (the ring may have passed its end since the slot)
          const uint32_t full = slot[p] < kr.at ? kr.phase : kr.phase ^ 1;
          if (!wait_bar(s, a, &s.kfull[slot[p]], full, 5u)) return;
        }
        const uint32_t i = (uint32_t)p * 2 + b;
        if (!wait_bar(s, a, &s.sempty[p][b], ((phase >> i) & 1) ^ 1, 6u)) return;
        phase ^= 1u << i;
        tc_fence_after();
        const uint64_t kd = k0 + (uint64_t)(slot[p] * (kTileBytes >> 4));
#pragma unroll
        for (int k8 = 0; k8 < 8; ++k8) {
          const uint64_t d = (uint64_t)((k8 >> 2) * (kHalf >> 4) + (k8 & 3) * 2);
          mma_bf16(tmem + i * 128u, kd + d, qd + d, idesc, k8 > 0 ? 1u : 0u);
        }
        mma_commit(&s.sfull[p][b]);
      }
      mma_commit(&s.qempty[qr.at]);
      qr.step();
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (p < nk) mma_commit(&s.kempty[slot[p]]);
  }
}

// The rows' references: those of the next two tiles are on their way.
__device__ __forceinline__ void refer(Smem& s, const WeighArgs& w, int lane) {
  const AttendArgs& a = w.a;
  ItemReader items;
  WeighItem it;
  // this lane's four rows of a tile: where their numbers are from the tile's first one's
  int64_t at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = lane + 32 * i, k = row / a.g;
    at[i] = (int64_t)k * a.h_q + row - k * a.g;
  }
  int t = 0;
  bool more = items.next(s, a, it, lane);
  if (more) t = it.tile0;
  auto look_up = [&](float (&to)[4]) {  // the next tile's; false: there is none
    if (!more) return false;
    const int rows = rows_of(w, it, t);
    const float* from = w.lse + (int64_t)(it.tok0 + t * w.tpt[it.source]) * a.h_q + it.head * a.g;
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = lane + 32 * i < rows ? from[at[i]] : -INFINITY;
    if (++t == it.tile0 + it.ntiles) {
      more = items.next(s, a, it, lane);
      if (more) t = it.tile0;
    }
    return true;
  };
  float even[4], odd[4];
  bool has_even = look_up(even), has_odd = look_up(odd);
  Ring<kRefs> r;
  auto put = [&](float (&x)[4], bool& has) {
    float ref[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ref[i] = weigh_ref(x[i]);
    has = look_up(x);
    if (!wait_warp(s, a, &s.rempty[r.at], r.phase ^ 1, 7u)) return false;
#pragma unroll
    for (int i = 0; i < 4; ++i) s.ref[r.at][lane + 32 * i] = ref[i];
    __syncwarp();
    if (lane == 0) mbar_arrive(&s.rfull[r.at]);
    r.step();
    return true;
  };
  while (has_even && put(even, has_even) && has_odd && put(odd, has_odd)) {
  }
}

__device__ __forceinline__ void add_up(Smem& s, const WeighArgs& w, uint32_t tmem, int tile, uint32_t parity) {
  const AttendArgs& a = w.a;
  const int lane = threadIdx.x & 31, row = threadIdx.x & 127, warp = row >> 5;
  const uint32_t ts = tmem + (uint32_t)(tile * 2 + parity) * 128u + ((uint32_t)(warp * 32) << 16);
  const uint64_t scale2 = pack_f32x2(a.scale_log2, a.scale_log2);
  const int k = tile * kKeys + row;
  ItemReader items;
  WeighItem next{};
  uint32_t n0 = 0, jobs = 0, merges = 0;  // row tiles before the item; this stream's products; items it has shared
  bool more = items.next(s, a, next, lane);
  auto page_of = [&](uint32_t n) {
    return more && (n & 1) == parity && k < next.nkeys ? weight_page(w, next, next.key0 + k) : 0;
  };
  int page = page_of(0);
  while (more) {
    const WeighItem it = next;
    const int j = it.key0 + k;
    // (the stream of the item's first tile has its keys' weights)
    const bool active = tile < key_tiles(it), mine = k < it.nkeys, first = (n0 & 1) == parity, both = it.ntiles > 1;
    // (on its way while the products are; the next item's page number too)
    float* at = mine && first && it.tile0 == 0 ? weight_at(w, it, j, page) : nullptr;
    const float before = weight_before(it, at, j);
    more = items.next(s, a, next, lane);
    page = page_of(n0 + (uint32_t)it.ntiles);
    float total = 0.f;
    const int tpt = w.tpt[it.source];
    for (int t = it.tile0; t < it.tile0 + it.ntiles; ++t, ++n0) {
      if ((n0 & 1) != parity) continue;
      const int rows = rows_of(w, it, t);
      // rows from this one on see the key
      const int from = it.source == 0 ? 0 : max((j - it.base - t * tpt) * a.g, 0);
      const uint32_t slot = n0 % kRefs;
      if (!wait_warp(s, a, &s.rfull[slot], (n0 / kRefs) & 1, 8u)) return;
      if (active) {
        if (!wait_warp(s, a, &s.sfull[tile][parity], jobs & 1, 9u)) return;
        ++jobs;
        tc_fence_after();
        float2 l = make_float2(0.f, 0.f);  // (more of them cost registers: two 47.0 us, four 47.9)
#pragma unroll 1
        for (int b = 0;; b += 32) {
          uint32_t x[32];
          tmem_ld_x32(ts + b, x);
          tmem_wait_ld();
          tmem_landed(x);
          const bool last = b + 32 >= rows;
          if (last) {  // the accumulator is read: the next product runs beside these columns
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sempty[tile][parity]);
          }
          if (b + 32 > rows) {  // (columns without a row hold anything)
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (b + c >= rows) x[c] = 0xff800000u;  // -inf
          }
          if (__any_sync(0xffffffffu, from > b)) {
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (b + c < from) x[c] = 0xff800000u;
          }
          const float4* ref = reinterpret_cast<const float4*>(s.ref[slot] + b);
#pragma unroll
          for (int c = 0; c < 32; c += 4) {
            const float4 f = ref[c / 4];
            fma_pair(x[c], x[c + 1], scale2, f.x, f.y);
            fma_pair(x[c + 2], x[c + 3], scale2, f.z, f.w);
            add_pair(l.x, l.y, ex2(__uint_as_float(x[c])), ex2(__uint_as_float(x[c + 1])));
            add_pair(l.x, l.y, ex2(__uint_as_float(x[c + 2])), ex2(__uint_as_float(x[c + 3])));
          }
          if (last) break;
        }
        total += l.x + l.y;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.rempty[slot]);
    }
    if (active && both) {
      // (warps of the same keys wait for each other only, each time in both directions, so
      // that neither's wait meets another phase)
      if (!first) {
        s.sum[tile][row] = total;
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.mready[tile][warp]);
        if (!wait_warp(s, a, &s.mdone[tile][warp], merges & 1, 11u)) return;
      } else {
        if (!wait_warp(s, a, &s.mready[tile][warp], merges & 1, 11u)) return;
        total += s.sum[tile][row];
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.mdone[tile][warp]);
      }
      ++merges;
    }
    if (at != nullptr) *at = weight_after(w, before, total);
    if (mine && first && it.tile0 != 0) w.next[(int64_t)blockIdx.x * kWeighSpan + k] = total;
  }
}

__global__ void __launch_bounds__(kThreads, 1)
    weigh_tc_kernel(const __grid_constant__ Maps m, const __grid_constant__ WeighArgs w) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];  // (as the swizzled tiles want; no room to round up)
  Smem& s = *reinterpret_cast<Smem*>(smem_raw);
  const AttendArgs& a = w.a;
  if ((smem_u32(smem_raw) & 1023u) != 0) {
    grid_wait();
    if (threadIdx.x == 0) {
      note(a, ECOKV_ERR_CUDA, 0u);
      w.next_item[blockIdx.x] = WeighItem{};  // (nothing to join)
    }
    return;
  }
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kKeyTiles; ++i) {
      mbar_init(&s.kfull[i], 1);
      mbar_init(&s.kempty[i], 1);
    }
    for (int i = 0; i < kRowTiles; ++i) {
      mbar_init(&s.qfull[i], 1);
      mbar_init(&s.qempty[i], 1);
    }
    for (int i = 0; i < kRefs; ++i) {
      mbar_init(&s.rfull[i], 1);
      mbar_init(&s.rempty[i], 8);  // the warps of a parity's streams
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s.sfull[i >> 1][i & 1], 1);
      mbar_init(&s.sempty[i >> 1][i & 1], 4);
    }
    for (int i = 0; i < 8; ++i) {
      mbar_init(&s.mready[i >> 2][i & 3], 1);
      mbar_init(&s.mdone[i >> 2][i & 3], 1);
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&s.ifull[i], 1);
      mbar_init(&s.iempty[i], 19);  // the warps of the copies, products and references, and the streams
    }
    mbar_init(&s.drained, 1);
    s.abort = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane < 4) tma_prefetch_desc(&m.q[0] + lane);
  if (warp == 3) {
    tmem_alloc(&s.tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // (what is above runs beside the end of the grid before)
  grid_wait();
  const uint32_t tmem = s.tmem;
  Issued d;
  if (warp >= 4) {
    add_up(s, w, tmem, (warp - 4) >> 3, ((warp - 4) >> 2) & 1);
  } else if (warp == 0) {
    // (the injected stall: no tile ever comes)
    if (a.stall == 0) produce(s, w, m, lane, d);
  } else if (warp == 1) {
    if (elect_one()) {
      multiply(s, w, tmem);
      mma_commit(&s.drained);
    }
  } else if (warp == 3) {
    refer(s, w, lane);
  } else {
    WeighWalk walk;
    walk.begin(w, blockIdx.x, lane, blockIdx.x == 0);
    Ring<kItems> r;
    for (bool first = true;; first = false) {
      WeighItem it{};
      const bool more = walk.next(w, it);
      if (first && lane == 0) w.next_item[blockIdx.x] = it;
      if (!wait_warp(s, a, &s.iempty[r.at], r.phase ^ 1, 10u)) break;
      if (lane == 0) {
        s.items[r.at] = it;
        mbar_arrive(&s.ifull[r.at]);
      }
      __syncwarp();
      r.step();
      if (!more) break;
    }
  }
  __syncwarp();
  // every MMA has completed (a CTA that gave up: those that it had issued)
  if (warp == 1) drain_bar(&s.drained, 0u);
  if (warp == 0) {
    // ... and every copy has landed: the last of each buffer's, should no one have waited for it
    for (uint32_t i = 0; i < kKeyTiles; ++i)
      if (d.k > i) drain_bar(&s.kfull[i], ((d.k - 1 - i) / kKeyTiles) & 1);
    for (uint32_t i = 0; i < kRowTiles; ++i)
      if (d.q > i) drain_bar(&s.qfull[i], ((d.q - 1 - i) / kRowTiles) & 1);
  }
  __syncthreads();
  // (a CTA that gave up leaves no sum: what lies there may be another call's)
  if (s.abort != 0 && tid < kWeighSpan) w.next[(int64_t)blockIdx.x * kWeighSpan + tid] = 0.f;
  grid_trigger();
  if (warp == 3) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

std::atomic<bool> g_attr_set[64];

}  // namespace

cudaError_t launch_weigh_tc(const WeighArgs& w, cudaStream_t st) {
  const AttendArgs& a = w.a;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  Maps m;
  for (int k = 0; k < 2; ++k) {
    const uint64_t dims[3] = {kD, (uint64_t)a.h_q, (uint64_t)a.tokens};
    const int64_t strides[2] = {a.q_head, a.q_token};
    const uint32_t box[3] = {64, (uint32_t)a.g, (uint32_t)w.tpt[k]};
    if (!map_of(&m.q[k], a.q, 3, dims, strides, box)) return cudaErrorInvalidValue;
  }
  m.pk = m.ck = m.q[0];  // that of a source that is not there is not used
  if (a.prefix.rows > 0) {
    const bool off = a.prefix.head_off != nullptr;
    const uint64_t dims[3] = {kD, (uint64_t)a.prefix.rows, off ? 1 : (uint64_t)a.h_kv};
    const int64_t strides[2] = {a.prefix.row_stride, off || a.h_kv == 1 ? a.prefix.row_stride : a.prefix.head_stride};
    const uint32_t box[3] = {64, kKeys, 1};
    if (!map_of(&m.pk, a.prefix.k, 3, dims, strides, box)) return cudaErrorInvalidValue;
  }
  if (a.has_cache) {
    const ecokv_pages& c = a.cache;
    const uint64_t dims[4] = {kD, (uint64_t)c.page_size, (uint64_t)a.h_kv, (uint64_t)c.n_pages};
    const int64_t strides[3] = {c.slot_stride, c.head_stride, c.page_stride};
    const uint32_t box[4] = {64, (uint32_t)(c.page_size < kKeys ? c.page_size : kKeys), 1, 1};
    if (!map_of(&m.ck, c.k, 4, dims, strides, box)) return cudaErrorInvalidValue;
  }
  const int smem = (int)sizeof(Smem);
  if (!g_attr_set[dev].load()) {  // a racing thread repeats the idempotent setting
    e = cudaFuncSetAttribute(weigh_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    g_attr_set[dev].store(true);
  }
  return launch_behind(weigh_tc_kernel, (unsigned)a.P, kThreads, (size_t)smem, st, m, w);
}

}  // namespace ecokv
