// Shared by the kernels that weigh keys (weigh_simt.cu, weigh_tc.cu, weigh_api.cu): how
// the work is cut and dealt.
//
// The attention's cut (attend.cuh) with the factors in each other's place: an item is one KV
// head and up to `span` consecutive keys of one source (the shared prefix or one
// sequence's slots), and its tiles are row tiles: up to tpt tokens with the query heads of the
// group, of all sequences (prefix) or of the item's own.  A key's sum then stays in
// a thread's register over all the rows that see it, the keys are read once and the few
// queries again for each item, from the L2.  All items' tiles in a row (the prefix's by
// head, the own ones by head and sequence) are dealt to the CTAs in equal runs of
// units: `lead` for an item's keys, `unit` for each of its tiles.  An item of more than
// `whole` units may be cut: its first CTA adds its sum to the weight, the others leave theirs,
// which a second kernel adds in their order.  A smaller one is its first unit's CTA's: it
// takes less time than that kernel's launch.
#pragma once

#include "attend.cuh"

namespace ecokv {

constexpr int kWeighSpan = 256;  // most keys an item has
constexpr int kMaxWeighCtas = 2 * kMaxAttendSms;

struct WeighItem {
  int source, head, seq;  // as in Item
  int key0, nkeys;        // its keys
  int tok0, ntok;         // tokens that see them: of the call, or of the sequence
  int base;               // token k sees keys up to base + k of the source (prefix: all)
  int row0;               // first row of the head's prefix (head_off)
  int tile0, ntiles;      // this CTA's row tiles
};

struct WeighArgs {
  AttendArgs a;           // tensors and sizes (out, lse and what follows tpt are not used)
  ecokv_weights pw, w;    // of the prefix, of the slots
  const float* lse;
  float decay;
  int span, span_log2, tpt[2], unit[2], lead, whole, least;
  float* next;            // [P][kWeighSpan] sums of the item that a CTA goes on with
  WeighItem* next_item;   // [P], tile0 = 0: none
};

// Row tiles of an item that so many tokens see (one at least, so that it is met).
__device__ __forceinline__ int row_tiles(const WeighArgs& w, int source, int ntok) {
  return ntok > w.tpt[source] ? (ntok - 1) / w.tpt[source] + 1 : 1;
}
__device__ __forceinline__ int weigh_per(const WeighArgs& w, int source, int ntok) {
  return w.lead + row_tiles(w, source, ntok) * w.unit[source];
}
// (31 bits hold it, as the host has checked for any of the call's sequences)
__device__ __forceinline__ int weigh_units(const WeighArgs& w, int source, int keys, int ntok) {
  return ((keys + w.span - 1) >> w.span_log2) * weigh_per(w, source, ntok);
}

// Tokens of the call that are of a sequence, from 0 on.
__device__ __forceinline__ int live_tokens(const AttendArgs& a) {
  return a.has_cache && a.starts != nullptr ? min(max(a.starts[a.batch], 0), a.tokens) : a.tokens;
}

// A warp's walk over its CTA's run of units, item by item.  Every lane holds the same
// state but for the 32 sequences (or heads) at hand, one a lane.
struct WeighWalk {
  int x, end, prefix_total, own;
  int live, lane;
  int b0, head;
  int left;    // keys of the head and sequence behind the item before, if that was met to its end
  int before;  // units of the sequences before b0
  WeighItem it;  // the one at hand, from which the next one of its head and sequence follows
  Seq s;
  int n, upto;

  __device__ __forceinline__ void chunk(const WeighArgs& w, int from, bool report) {
    b0 = from;
    s = Seq{0, 0, 0};
    n = 0;
    if (b0 + lane < w.a.batch) {
      s = load_seq(w.a, b0 + lane, report);
      n = weigh_units(w, 1, s.L, s.T);
    }
    upto = Walk::scan(n, lane);  // (may wrap where begin() drops the sequences)
  }

  // All of the warp's lanes; `report`: note what is out of range.
  __device__ __forceinline__ void begin(const WeighArgs& w, int cta, int lane_, bool report) {
    const AttendArgs& a = w.a;
    lane = lane_;
    live = live_tokens(a);
    prefix_total = 0;
    if (a.prefix.rows > 0) {
      if (a.prefix.head_off == nullptr) {
        prefix_total = a.h_kv * weigh_units(w, 0, a.prefix.rows, live);
      } else {
#pragma unroll 1
        for (int h0 = 0; h0 < a.h_kv; h0 += 32) {
          int row0, v = 0;
          if (h0 + lane < a.h_kv) v = weigh_units(w, 0, prefix_rows(a, h0 + lane, row0, report), live);
          prefix_total += (int)__reduce_add_sync(0xffffffffu, (unsigned)v);
        }
      }
    }
    own = 0;
    if (a.has_cache) {
      chunk(w, 0, report);
      long long sum = n;
#pragma unroll 4
      for (int b = 32 + lane; b < a.batch; b += 32) {
        const Seq q = load_seq(a, b, report);
        sum += weigh_units(w, 1, q.L, q.T);
      }
      // (in 64 bits: starts that overlap may have every sequence hold all of the tokens)
      const unsigned most = (unsigned)min(sum, 0x7fffffffll);
      sum = __reduce_add_sync(0xffffffffu, most & 0xffffu) +
            ((long long)__reduce_add_sync(0xffffffffu, most >> 16) << 16);
      if (sum * a.h_kv > 0x7fffffff - prefix_total) {
        if (report && lane == 0) note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)a.batch);
        sum = 0;
      }
      own = (int)sum;
    }
    before = 0;
    head = 0;
    left = 0;
    const int total = prefix_total + a.h_kv * own;
    const int run = max((int)(((unsigned)total + (unsigned)a.P - 1u) / (unsigned)a.P), w.least);
    x = (int)min((unsigned)cta * (unsigned)run, (unsigned)total);
    end = (int)min((unsigned)x + (unsigned)run, (unsigned)total);
  }

  // The next item (the same in every lane); false: none left, and `to` as it was.
  __device__ __forceinline__ bool next(const WeighArgs& w, WeighItem& to) {
#pragma unroll 1
    while (x < end) {
      if (!at(w)) return false;
      if (it.ntiles > 0) {
        to = it;
        return true;
      }
    }
    return false;
  }
  // The part of an item from unit x on, which may be less than its first tile (ntiles <= 0).
  __device__ __forceinline__ bool at(const WeighArgs& w) {
    const AttendArgs& a = w.a;
    int y, keys;
    if (left > 0) {  // the item behind the one before
      it.key0 += w.span;
      it.nkeys = min(left, w.span);
      return part(w, 0, left);
    }
    if (x < prefix_total) {
      it.source = 0;
      it.seq = 0;
      it.row0 = 0;
      it.tok0 = 0;
      it.ntok = live;
      if (a.prefix.head_off == nullptr) {
        keys = a.prefix.rows;
        const int per = prefix_total / a.h_kv;
        it.head = x / per;
        y = x - it.head * per;
      } else {
        int at = 0;
#pragma unroll 1
        for (int h0 = 0;; h0 += 32) {
          if (h0 >= a.h_kv) return false;  // (only when the offsets change under the kernel; so below)
          int r0 = 0, rows = 0;
          if (h0 + lane < a.h_kv) rows = prefix_rows(a, h0 + lane, r0, false);
          const int v = weigh_units(w, 0, rows, live), up = Walk::scan(v, lane);
          const int all = __shfl_sync(0xffffffffu, up, 31);
          if (x < at + all) {
            const int l = __ffs(__ballot_sync(0xffffffffu, x < at + up)) - 1;
            it.head = h0 + l;
            y = x - at - __shfl_sync(0xffffffffu, up - v, l);
            it.row0 = __shfl_sync(0xffffffffu, r0, l);
            keys = __shfl_sync(0xffffffffu, rows, l);
            break;
          }
          at += all;
        }
      }
      it.base = keys;
    } else {
      y = x - prefix_total;
      const int h = y / own;
      y -= h * own;
      if (h != head && b0 != 0) {
        before = 0;
        chunk(w, 0, false);
      }
      head = h;
      int all;
#pragma unroll 1
      while (y >= before + (all = __shfl_sync(0xffffffffu, upto, 31))) {
        before += all;
        if (b0 + 32 >= a.batch) return false;
        chunk(w, b0 + 32, false);
      }
      const int l = __ffs(__ballot_sync(0xffffffffu, y < before + upto)) - 1;
      y -= before + __shfl_sync(0xffffffffu, upto - n, l);
      keys = __shfl_sync(0xffffffffu, s.L, l);
      it.source = 1;
      it.head = h;
      it.seq = b0 + l;
      it.row0 = 0;
      it.tok0 = __shfl_sync(0xffffffffu, s.start, l);
      it.ntok = __shfl_sync(0xffffffffu, s.T, l);
      it.base = keys - it.ntok;
    }
    const int per = weigh_per(w, it.source, it.ntok), i = y / per;
    it.key0 = i * w.span;
    it.nkeys = min(keys - it.key0, w.span);
    return part(w, y - i * per, keys - it.key0);
  }
  // The tiles of an item whose first unit lies within this CTA's part of it, y .. z - 1; the
  // item and what lies behind it of its head and sequence have `keys` keys.
  __device__ __forceinline__ bool part(const WeighArgs& w, int y, int keys) {
    const int per = weigh_per(w, it.source, it.ntok), u = w.unit[it.source];
    const bool whole = per <= w.whole;
    const int z = whole ? per : min(per, y + end - x);
    it.tile0 = (max(y - w.lead, 0) + u - 1) / u;
    it.ntiles = whole && y > 0 ? 0 : (max(z - w.lead, 0) + u - 1) / u - it.tile0;
    x += z - y;
    left = z == per ? max(keys - w.span, 0) : 0;
    return z > y && keys > 0;  // (else nothing would move on)
  }
};

// Where the weight of key j of the item's source is, whose page is `page`; NULL: a slot without
// a page.
__device__ __forceinline__ int weight_page(const WeighArgs& w, const WeighItem& it, int j) {
  const AttendArgs& a = w.a;
  return it.source == 0 ? 0 : a.cache.table[(int64_t)it.seq * a.cache.table_stride + (j >> a.page_shift)];
}
__device__ __forceinline__ float* weight_at(const WeighArgs& w, const WeighItem& it, int j, int page) {
  const AttendArgs& a = w.a;
  if (it.source == 0)
    return w.pw.w + (a.prefix.head_off ? 0 : (int64_t)it.head * w.pw.head_stride) +
           ((int64_t)it.row0 + j) * w.pw.slot_stride;
  if (page < 0 || page >= a.cache.n_pages) {
    note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)it.seq);
    return nullptr;
  }
  return w.w.w + (int64_t)page * w.w.page_stride + (int64_t)it.head * w.w.head_stride +
         (int64_t)(j & (a.cache.page_size - 1)) * w.w.slot_stride;
}
__device__ __forceinline__ float* weight_at(const WeighArgs& w, const WeighItem& it, int j) {
  return weight_at(w, it, j, weight_page(w, it, j));
}
// The weight that the item's sum is added to: a new token's own slot starts at 0.
__device__ __forceinline__ float weight_before(const WeighItem& it, const float* at, int j) {
  return at == nullptr || (it.source != 0 && j >= it.base) ? 0.f : *at;
}
// (what was before may be anything where nothing of it counts)
__device__ __forceinline__ float weight_after(const WeighArgs& w, float before, float sum) {
  return w.decay == 0.f ? sum : fmaf(w.decay, before, sum);
}
// What a row's scores (in log2 units) are taken relative to, negated: rows that saw no key
// give nothing.
__device__ __forceinline__ float weigh_ref(float lse) { return lse == -INFINITY ? -INFINITY : -lse * 1.4426950408889634f; }

cudaError_t launch_weigh_simt(const WeighArgs& w, ecokv_dtype dt, cudaStream_t st);
cudaError_t launch_weigh_tc(const WeighArgs& w, cudaStream_t st);

}  // namespace ecokv
