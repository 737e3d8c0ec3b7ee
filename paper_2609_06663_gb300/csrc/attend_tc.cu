// Attention of the decode step on the tensor cores (bf16): items and tiles as in
// attend.cuh, one persistent CTA an SM.
//
// A row tile is 128 rows = tpt tokens x g query heads of one KV head, the M of both
// products.  S = Q K^T goes to tensor memory, a thread a row takes it through the
// softmax and leaves the weights there as bf16, from where the second product O +=
// P V reads them; O stays in tensor memory through the item.  Two warpgroups ("streams") do
// the softmax of alternating jobs, so that one's exponentials run beside the
// other's products: the jobs of an item are its two row tiles on each key tile, or, with
// one row tile, the key tiles in turn, whose sums are added at its end.
// Weights refer to the maximum of the row's first 32 keys, and to another only when a
// score exceeds it by 2^kRaise: bf16 has the range of fp32 and no weight is more
// exact for being below one, so that a tile needs no pass for its maximum.
// The weights are rounded to bf16 because both factors of an MMA have one type and V
// is bf16; they are summed before that, in fp32.  Each is off by 2^-9 at most, the
// output by 2.2 to 2.4e-3 relative where one rounding of an exact output is 1.7e-3.  (A
// further product with what the rounding left would double the second one's work.)
//
// Warps: 0 copies (TMA; a lane a page), 1 and 3 the streams' products, 2 the walk over
// the items, 4-7 and 8-11 the streams' softmax.

#include <atomic>

#include "attend.cuh"
#include "decode_ptx.cuh"
#include "tc_tile.cuh"

namespace ecokv {
namespace {

using namespace ptx;

constexpr int kThreads = 384;
constexpr int kStages = 5;          // tiles of K or V in the ring
constexpr int kItems = 4;           // items ahead of their consumers
constexpr uint32_t kHalf = kTileBytes / 2;  // 128 rows x 64 columns
// log2 units: weights up to 2^16, so that a sum of 2^25 of them (the prefix's keys and a
// sequence's own) with values below 2^86 stays below 2^127
constexpr float kRaise = 16.f;

struct Smem {
  uint8_t q[2][kTileBytes];
  uint8_t ring[kStages][kTileBytes];
  // A tile's arrival is signalled to those who use it, on a barrier that no other
  // tile of the stage is signalled on: to stream 0, to stream 1 or (2) to both.
  // (A wait tells a phase from its neighbours by its parity only, so whoever waits on a
  // barrier has to see each of its phases.)
  uint64_t full[3][kStages], empty[kStages];
  uint64_t qfull[2], qempty[2];
  uint64_t sfull[2], vready[2], pready[2], ofull[2];
  uint64_t mready[4], mdone[4];  // between the streams' warps of the same rows
  float2 ml[128];                // the second stream's references and sums, by row
  uint64_t ifull[kItems], iempty[kItems];
  uint64_t drained;
  Item items[kItems];
  uint32_t tmem;
  volatile int abort;
};

static_assert(sizeof(Smem) + 1024 <= 232448, "one CTA's shared memory");

struct Maps {
  CUtensorMap q, pk, pv, ck, cv;
};

// Bounded wait: false once this CTA has given up.  (The clock is read every 16th
// try: reading it takes longer than a try.  One copy of this for all waits: inlined in
// each, it was a fifth of the kernel's code.)
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

// The next item of the queue, for a warp; false: none left, or given up.
struct ItemReader {
  uint32_t n = 0;
  __device__ __forceinline__ bool next(Smem& s, const AttendArgs& a, Item& it, int lane) {
    const uint32_t e = n % kItems;
    if (!wait_warp(s, a, &s.ifull[e], (n / kItems) & 1, 1u)) return false;
    it = s.items[e];
    __syncwarp();
    if (lane == 0) mbar_arrive(&s.iempty[e]);
    ++n;
    return it.ntiles > 0;
  }
};

__device__ __forceinline__ void store8(float* p, const uint32_t* r) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// What has been issued, for those who wait for it to land.
struct Issued {
  uint32_t load = 0, ql = 0;  // tiles of K and V, and of Q
  uint32_t phase[3] = {0, 0, 0};  // bit st: the parity of full[.][st]'s next phase
  uint32_t kind[kStages] = {};    // the stage's last: index of its barrier
};

__device__ __forceinline__ void produce(Smem& s, const AttendArgs& a, const Maps& m, int lane, Issued& d) {
  ItemReader items;
  Item it;
  uint32_t n0 = 0;  // jobs before the item
  const int q_bytes = a.tpt * a.g * 256;
  while (items.next(s, a, it, lane)) {
    const int nq = it.ntok > a.tpt ? 2 : 1;
    for (int r = 0; r < nq; ++r) {
      const int slot = d.ql & 1;
      if (!wait_warp(s, a, &s.qempty[slot], ((d.ql >> 1) & 1) ^ 1, 2u)) return;
      if (lane == 0) mbar_expect_tx(&s.qfull[slot], (uint32_t)q_bytes);
      __syncwarp();
      if (lane < 2)
        tma_load_3d(s.q[slot] + lane * kHalf, &m.q, &s.qfull[slot], lane * 64, it.head * a.g, it.tok0 + r * a.tpt);
      ++d.ql;
    }
    // what this lane copies of a tile: half the columns of the prefix's rows, or a page of it
    const bool own = it.source != 0;
    const int head = own || a.prefix.head_off == nullptr ? it.head : 0;
    const uint32_t box = own ? (uint32_t)min(a.cache.page_size, kKeys) : kKeys;
    const uint32_t at = own ? (((uint32_t)lane << a.page_shift) & (kKeys - 1)) * 128u : lane * kHalf;
    const int* table = a.cache.table + (int64_t)it.seq * a.cache.table_stride;
    int c0 = 0, n = 2, page = 0;
    auto look_up = [&](int t) {  // this lane's page of tile t, ahead of its turn
      const int from = t * kKeys, to = min(from + kKeys, it.vis);
      c0 = from >> a.page_shift;
      n = ((to - 1) >> a.page_shift) - c0 + 1;
      if (lane < n) page = table[c0 + lane];
    };
    if (own) look_up(it.tile0);
    for (int t = it.tile0; t < it.tile0 + it.ntiles; ++t) {
      const int row = own ? (t * kKeys) & (a.cache.page_size - 1) : it.row0 + t * kKeys;
      const int copies = n, z = page;
      const uint32_t kind = nq == 2 ? 2u : (n0 + (uint32_t)(t - it.tile0)) & 1;
      const bool bad = own && lane < copies && (z < 0 || z >= a.cache.n_pages);
      if (bad) note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)it.seq);
      const int w = bad ? a.cache.n_pages : z;  // out of the map's bounds: zeros
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const uint32_t st = d.load % kStages;
        if (!wait_warp(s, a, &s.empty[st], ((d.load / kStages) & 1) ^ 1, 3u)) return;
        uint8_t* dst = s.ring[st] + at;
        uint64_t* bar = &s.full[kind][st];
#pragma unroll
        for (uint32_t i = 0; i < 3; ++i) d.phase[i] ^= i == kind ? 1u << st : 0u;
#pragma unroll
        for (uint32_t i = 0; i < kStages; ++i) d.kind[i] = i == st ? kind : d.kind[i];
        if (lane == 0) mbar_expect_tx(bar, own ? box * copies * 256u : kTileBytes);
        __syncwarp();
        if (lane < copies) {
          if (own) {
            tma_load_4d(dst, kv == 0 ? &m.ck : &m.cv, bar, 0, row, head, w);
            tma_load_4d(dst + kHalf, kv == 0 ? &m.ck : &m.cv, bar, 64, row, head, w);
          } else {
            tma_load_3d(dst, kv == 0 ? &m.pk : &m.pv, bar, lane * 64, row, head);
          }
        }
        ++d.load;
        if (kv == 0 && own && t + 1 < it.tile0 + it.ntiles) look_up(t + 1);
      }
    }
    n0 += (uint32_t)(it.ntiles * nq);
  }
}

// The products of one stream, by one thread: the first of a job, then, when its
// weights are there, the second, while the other stream's thread keeps the tensor pipe
// busy.  (One thread for both streams took 2500 cycles a job: every wait stood
// between products that had nothing to do with it.)
__device__ __forceinline__ void multiply(Smem& s, const AttendArgs& a, uint32_t tmem, uint32_t stream) {
  constexpr uint32_t idesc1 = idesc_bf16(128, 128, false, false), idesc2 = idesc_bf16(128, 128, false, true);
  const uint32_t ts = tmem + stream * 256u, to = ts + 128u;  // scores, later the weights; the sum
  uint32_t n0 = 0, load = 0, ql = 0, k = 0;  // jobs before the item, tiles of K and V, of Q; this stream's jobs
  uint32_t phase[2] = {0, 0};  // bit st: parity of the next phase of this stream's full[.][st], of both streams'
  for (uint32_t e = 0;; ++e) {
    if (!wait_bar(s, a, &s.ifull[e % kItems], (e / kItems) & 1, 1u)) return;
    const int left = s.items[e % kItems].vis - s.items[e % kItems].tile0 * kKeys;  // keys from its first tile on
    const int ntiles = s.items[e % kItems].ntiles;
    const bool two = s.items[e % kItems].ntok > a.tpt;
    mbar_arrive(&s.iempty[e % kItems]);
    if (ntiles <= 0) return;
    const uint32_t p = (stream ^ n0) & 1, q = ql + (two ? p : 0);  // its row tile, or its key tiles in turn
    // Every buffer is released by two arrivals: one of each stream for Q and, with two
    // row tiles, for K and V; with one row tile both of the key tile's stream.
    for (uint32_t x = ql; x < ql + (two ? 2u : 1u); ++x) {
      if (!wait_bar(s, a, &s.qfull[x & 1], (x >> 1) & 1, 6u)) return;
      if (x != q) mbar_arrive(&s.qempty[x & 1]);
    }
    const uint64_t qd = smem_desc(smem_u32(s.q[q & 1]), 16, 1024, 2);
    const int step = two ? 1 : 2, t0 = two ? 0 : (int)p;
    uint64_t* full = s.full[two ? 2u : stream];
    uint32_t ph = two ? phase[1] : phase[0];
    for (int t = t0; t < ntiles; t += step, ++k) {
      const uint32_t sk = (load + 2 * t) % kStages, sv = (load + 2 * t + 1) % kStages;
      if (!wait_bar(s, a, &full[sk], (ph >> sk) & 1, 7u)) return;
      ph ^= 1u << sk;
      tc_fence_after();
      const uint64_t kd = smem_desc(smem_u32(s.ring[sk]), 16, 1024, 2);
#pragma unroll
      for (int k8 = 0; k8 < 8; ++k8) {
        const uint64_t d = (uint64_t)((k8 >> 2) * (kHalf >> 4) + (k8 & 3) * 2);
        mma_bf16(ts, qd + d, kd + d, idesc1, k8 > 0 ? 1u : 0u);
      }
      mma_commit(&s.sfull[stream]);
      mma_commit(&s.empty[sk]);
      if (!two) mma_commit(&s.empty[sk]);
      const int there = left - t * kKeys;  // keys of the tile
      if (!wait_bar(s, a, &full[sv], (ph >> sv) & 1, 4u)) return;
      ph ^= 1u << sv;
      if (there < kKeys) mbar_arrive(&s.vready[stream]);
      if (!wait_bar(s, a, &s.pready[stream], k & 1, 5u)) return;
      tc_fence_after();
      const uint64_t vd = smem_desc(smem_u32(s.ring[sv]), kHalf, 1024, 2);
      const int steps = min(there + 31, kKeys) >> 5;  // blocks of 32 keys that are there
#pragma unroll
      for (int k8 = 0; k8 < 8; ++k8)  // 16 keys a step
        if (k8 < 2 * steps)
          mma_bf16_ta(to, ts + k8 * 8u, vd + (uint64_t)(k8 * 128), idesc2, k8 > 0 || t > t0 ? 1u : 0u);
      mma_commit(&s.empty[sv]);
      if (!two) mma_commit(&s.empty[sv]);
    }
    if (two) phase[1] = ph;
    else phase[0] = ph;
    if (t0 < ntiles) {
      mma_commit(&s.ofull[stream]);
      mma_commit(&s.qempty[q & 1]);
    } else {
      mbar_arrive(&s.qempty[q & 1]);
    }
    load += 2 * (uint32_t)ntiles;
    n0 += (uint32_t)ntiles * (two ? 2u : 1u);
    ql += two ? 2u : 1u;
  }
}

__device__ __forceinline__ void soften(Smem& s, const AttendArgs& a, uint32_t tmem, int stream) {
  const int lane = threadIdx.x & 31, row = threadIdx.x & 127, warp = row >> 5;
  const uint32_t ts = tmem + (uint32_t)stream * 256u + ((uint32_t)(warp * 32) << 16), to = ts + 128u;
  const int row_k = row / a.g;
  const uint64_t scale2 = pack_f32x2(a.scale_log2, a.scale_log2);
  ItemReader items;
  Item it;
  // jobs and tiles before the item; this stream's jobs, items and ragged tiles
  uint32_t n0 = 0, tile_n = 0, k = 0, ends = 0, tails = 0;
  uint32_t merges = 0;  // items of which this warp's rows are in both streams
  while (items.next(s, a, it, lane)) {
    const bool two = it.ntok > a.tpt;
    const int p = (stream ^ (int)n0) & 1;  // which of the item's row tiles, or of its key tiles in turn
    const int tok = two ? p * a.tpt : 0;
    const int rows = min(it.ntok - tok, a.tpt) * a.g;
    const bool active = warp * 32 < rows;
    const int lim = it.lim0 + (tok + row_k) * it.slope;
    float m = -INFINITY;  // the reference
    float2 l[4];          // the sum of the weights, in eight parts
#pragma unroll
    for (int q = 0; q < 4; ++q) l[q] = make_float2(0.f, 0.f);
    const int step = two ? 1 : 2, t0 = two ? 0 : p;
    for (int t = t0; t < it.ntiles; t += step, ++k) {
      const int from = (it.tile0 + t) * kKeys;
      const int nv = it.vis - from;  // keys of the tile that are there (128 or more: all)
      if (!wait_warp(s, a, &s.sfull[stream], k & 1, 8u)) return;
      tc_fence_after();
      const int nc = min(nv + 31, kKeys) >> 5;  // blocks of 32 keys that are there
      if (active) {
        // Blocks of 32 keys in a loop that stays rolled: a call of a few tiles runs this
        // code but once or twice, and fetching code takes longer than running it (all
        // of a tile's scores in registers and unrolled: the batch of 16 over 3277 rows
        // 16.2 us, 1952 items of a tile each 59.0; in two rolled passes, one for the
        // maximum, 15.1 and 50.2; so 15.0 and 49.1, 16 questions of 61 tokens over 6554
        // rows 109.8 and not 116.6; with what came after it 14.7, 45.6 and 107)
        const int seen = lim - from;
#pragma unroll 1
        for (int b = 0; b < nc; ++b) {
          uint32_t x[32], w[16];
          tmem_ld_x32(ts + 32 * b, x);
          tmem_wait_ld();
          tmem_landed(x);
          const int here = seen - 32 * b;
          if (__any_sync(0xffffffffu, here < 32)) {
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (c >= here) x[c] = 0xff800000u;  // -inf
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 32; c += 8)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              mx[q] = fmaxf(fmaxf(mx[q], __uint_as_float(x[c + q])), __uint_as_float(x[c + 4 + q]));
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
          if (__any_sync(0xffffffffu, top > m + kRaise)) {
            // another reference, by a power of two (the first one as it is): what was
            // weighted by the old one follows.  (This stream's product before is
            // complete: it precedes this job's first in the tensor pipe.)
            float up = m, f = 1.f;
            if (top > m + kRaise) {
              up = m == -INFINITY ? top : m + ceilf(top - m);
              f = ex2(m - up);
            }
            m = up;
#pragma unroll
            for (int q = 0; q < 4; ++q) l[q] = make_float2(l[q].x * f, l[q].y * f);
            if (b > 0) {
              tmem_wait_st();
#pragma unroll 1
              for (int q = 0; q < b; ++q) {
                tmem_ld_x16(ts + 16 * q, w);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 16; ++c)
                  w[c] = pack_bf16x2(__uint_as_float(w[c] << 16) * f, __uint_as_float(w[c] & 0xffff0000u) * f);
                tmem_st_x16(ts + 16 * q, w);
              }
            }
            if (t > t0) {
#pragma unroll 1
              for (int c = 0; c < kD; c += 16) {
                tmem_ld_x16(to + c, w);
                tmem_wait_ld();
#pragma unroll
                for (int q = 0; q < 16; ++q) w[q] = __float_as_uint(__uint_as_float(w[q]) * f);
                tmem_st_x16(to + c, w);
              }
            }
          }
          const float nref = m == -INFINITY ? 0.f : -m;
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            fma_pair(x[c], x[c + 1], scale2, nref, nref);
            const float e0 = ex2(__uint_as_float(x[c])), e1 = ex2(__uint_as_float(x[c + 1]));
            add_pair(l[(c >> 1) & 3].x, l[(c >> 1) & 3].y, e0, e1);
            w[c / 2] = pack_bf16x2(e0, e1);
          }
          tmem_st_x16(ts + 16 * b, w);
        }
        tmem_wait_st();
      }
      if (nv < kKeys) {
        // rows of V past the keys that are there may hold anything, and 0 * NaN is NaN
        const uint32_t st = (2 * (tile_n + t) + 1) % kStages;
        if (!wait_warp(s, a, &s.vready[stream], tails & 1, 9u)) return;
        // (sixteen threads a row's two halves)
        for (int r = nv + (row >> 4); r < 32 * nc; r += 8)
          *reinterpret_cast<uint4*>(s.ring[st] + (row & 8 ? kHalf : 0u) + r * 128 + (row & 7) * 16) =
              make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async_smem();
        ++tails;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.pready[stream]);
    }
    // The row's sum.  Where the streams have had an item's key tiles in turn, the one
    // that had the first adds the other's sum to its own: a warp sees the tensor
    // memory of its rows in both.  (Warps of the same rows wait for each other only,
    // each time in both directions, so that neither's wait meets another phase.  Left
    // to the joining kernel, the two sums took 98.4 us and not 94.1 at 32 tokens over
    // 131072 rows.)
    const bool any = t0 < it.ntiles, both = !two && it.ntiles > 1;
    if (any && !wait_warp(s, a, &s.ofull[stream], ends & 1, 10u)) return;
    if (active && any) {
      tc_fence_after();
      float sum = ((l[0].x + l[0].y) + (l[1].x + l[1].y)) + ((l[2].x + l[2].y) + (l[3].x + l[3].y));
      if (both && p == 1) {
        s.ml[row] = make_float2(m, sum);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.mready[warp]);
        if (!wait_warp(s, a, &s.mdone[warp], merges & 1, 14u)) return;
        tc_fence_after();
      } else {
        float f = 1.f, f2 = 0.f;
        if (both) {
          if (!wait_warp(s, a, &s.mready[warp], merges & 1, 14u)) return;
          tc_fence_after();
          const float2 ml = s.ml[row];
          const float up = fmaxf(m, ml.x), ref = up == -INFINITY ? 0.f : up;
          f = ex2(m - ref);
          f2 = ex2(ml.x - ref);
          sum = fmaf(sum, f, ml.y * f2);
          m = up;
        }
        const bool first = it.tile0 == 0;
        const int token = it.tok0 + tok + row_k, hq = it.head * a.g + row - row_k * a.g;
        const size_t at = first ? first_row(a, it.source, token, hq) : next_row(a, blockIdx.x, p, row);
        float* dst = (first ? a.first_o : a.next_o) + at * kD;
        const bool mine = row < rows;
        if (mine) (first ? a.first_ml : a.next_ml)[at] = make_float2(m, sum);
        const uint32_t other = to ^ 256u;  // the other stream's sum of the same rows
#pragma unroll 1
        for (int c = 0; c < kD; c += 32) {
          uint32_t o[32], o2[32];
          tmem_ld_x32(to + c, o);
          if (both) tmem_ld_x32(other + c, o2);
          tmem_wait_ld();
          tmem_landed(o);
          if (both) {
            tmem_landed(o2);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              // (without weight it counts nothing, whatever it holds)
              const float own = f > 0.f ? __uint_as_float(o[j]) : 0.f, its = f2 > 0.f ? __uint_as_float(o2[j]) : 0.f;
              o[j] = __float_as_uint(fmaf(its, f2, own * f));
            }
          }
          if (mine) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) store8(dst + c + j, o + j);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (both && lane == 0) mbar_arrive(&s.mdone[warp]);
      }
    }
    if (active && both) ++merges;
    if (any) ++ends;
    tile_n += it.ntiles;
    n0 += it.ntiles * (two ? 2 : 1);
  }
}

__global__ void __launch_bounds__(kThreads, 1)
    attend_tc_kernel(const __grid_constant__ Maps m, const __grid_constant__ AttendArgs a) {
  extern __shared__ uint8_t smem_raw[];
  Smem& s = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      for (int k = 0; k < 3; ++k) mbar_init(&s.full[k][i], 1);
      mbar_init(&s.empty[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.qfull[i], 1);
      mbar_init(&s.qempty[i], 2);
      mbar_init(&s.sfull[i], 1);
      mbar_init(&s.vready[i], 1);
      mbar_init(&s.pready[i], 4);
      mbar_init(&s.ofull[i], 1);
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&s.ifull[i], 1);
      mbar_init(&s.iempty[i], 11);  // the warps of the copies, the MMAs and the streams
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s.mready[i], 1);
      mbar_init(&s.mdone[i], 1);
    }
    mbar_init(&s.drained, 2);
    s.abort = 0;
    fence_mbar_init();
  }
  if (warp == 0 && lane < 5) tma_prefetch_desc(&m.q + lane);
  if (warp == 3) {
    tmem_alloc(&s.tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // (what is above runs beside the end of the grid before)
  grid_wait();
  Walk w;
  if (warp == 2) w.begin(a, blockIdx.x, lane);
  const uint32_t tmem = s.tmem;
  Issued d;
  if (warp >= 4) {
    soften(s, a, tmem, (warp >> 2) - 1);
  } else {
    if (warp == 0) {
      // (the injected stall: no tile ever comes)
      if (a.stall == 0) produce(s, a, m, lane, d);
    } else if (warp == 1 || warp == 3) {
      if (lane == 0) {
        multiply(s, a, tmem, (uint32_t)warp >> 1);
        mma_commit(&s.drained);
      }
      __syncwarp();
    } else if (warp == 2) {
      for (uint32_t n = 0;; ++n) {
        Item it;
        const bool more = w.next(a, it);
        if (!more) it.ntiles = 0;
        if (!wait_warp(s, a, &s.iempty[n % kItems], ((n / kItems) & 1) ^ 1, 11u)) break;
        if (lane == 0) {
          s.items[n % kItems] = it;
          mbar_arrive(&s.ifull[n % kItems]);
        }
        __syncwarp();
        if (!more) break;
      }
    }
  }
  __syncwarp();
  // every MMA has completed (a CTA that gave up: those that it had issued)
  if (warp == 1 || warp == 3) drain_bar(&s.drained, 0u);
  if (warp == 0) {
    // ... and every copy has landed: the last of each buffer's, should no one have waited for it
#pragma unroll
    for (uint32_t i = 0; i < kStages; ++i)
      if (d.load > i) {
        const uint32_t k = d.kind[i], next = k == 0 ? d.phase[0] : k == 1 ? d.phase[1] : d.phase[2];
        drain_bar(&s.full[k][i], ((next >> i) & 1) ^ 1);
      }
    for (uint32_t i = 0; i < 2; ++i)
      if (d.ql > i) drain_bar(&s.qfull[i], ((d.ql - 1 - i) / 2) & 1);
  }
  __syncthreads();
  // (triggered at the start, the joining kernel's launch took 2 us longer)
  grid_trigger();
  if (warp == 3) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

std::atomic<bool> g_attr_set[64];

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static std::atomic<EncodeTiledFn> fn{nullptr};  // a racing thread repeats the lookup
  EncodeTiledFn f = fn.load();
  if (f == nullptr) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess) {
      f = reinterpret_cast<EncodeTiledFn>(p);
      fn.store(f);
    }
  }
  return f;
}

// A tensor of bf16 rows of 128, the axes after the first `strides` elements apart, in
// boxes of 64 columns with the 128-byte swizzle.
bool map_of(CUtensorMap* m, const void* base, int rank, const uint64_t* dims, const int64_t* strides,
            const uint32_t* box) {
  const EncodeTiledFn enc = encode_fn();
  cuuint64_t d[4], st[3];
  cuuint32_t b[4];
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    d[i] = dims[i];
    b[i] = box[i];
    if (i > 0) st[i - 1] = (cuuint64_t)strides[i - 1] * 2;
  }
  return enc != nullptr &&
         enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d, st, b, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  Maps m;
  {
    const uint64_t dims[3] = {kD, (uint64_t)a.h_q, (uint64_t)a.tokens};
    const int64_t strides[2] = {a.q_head, a.q_token};
    const uint32_t box[3] = {64, (uint32_t)a.g, (uint32_t)a.tpt};
    if (!map_of(&m.q, a.q, 3, dims, strides, box)) return cudaErrorInvalidValue;
  }
  m.pk = m.pv = m.ck = m.cv = m.q;  // those of a source that is not there are not used
  if (a.prefix.rows > 0) {
    const bool off = a.prefix.head_off != nullptr;
    const uint64_t dims[3] = {kD, (uint64_t)a.prefix.rows, off ? 1 : (uint64_t)a.h_kv};
    const int64_t strides[2] = {a.prefix.row_stride, off || a.h_kv == 1 ? a.prefix.row_stride : a.prefix.head_stride};
    const uint32_t box[3] = {64, kKeys, 1};
    if (!map_of(&m.pk, a.prefix.k, 3, dims, strides, box) || !map_of(&m.pv, a.prefix.v, 3, dims, strides, box))
      return cudaErrorInvalidValue;
  }
  if (a.has_cache) {
    const ecokv_pages& c = a.cache;
    const uint64_t dims[4] = {kD, (uint64_t)c.page_size, (uint64_t)a.h_kv, (uint64_t)c.n_pages};
    const int64_t strides[3] = {c.slot_stride, c.head_stride, c.page_stride};
    const uint32_t box[4] = {64, (uint32_t)(c.page_size < kKeys ? c.page_size : kKeys), 1, 1};
    if (!map_of(&m.ck, c.k, 4, dims, strides, box) || !map_of(&m.cv, c.v, 4, dims, strides, box))
      return cudaErrorInvalidValue;
  }
  const int smem = (int)sizeof(Smem) + 1024;
  if (!g_attr_set[dev].load()) {  // a racing thread repeats the idempotent setting
    e = cudaFuncSetAttribute(attend_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    g_attr_set[dev].store(true);
  }
  return launch_behind(attend_tc_kernel, (unsigned)a.P, kThreads, (size_t)smem, st, m, a);
}

}  // namespace ecokv
