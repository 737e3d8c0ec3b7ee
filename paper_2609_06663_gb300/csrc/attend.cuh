// Shared by the attention kernels of the decode step (attend_simt.cu, attend_tc.cu,
// attend_api.cu): how the work is cut into items and tiles, and where partial
// sums go.
//
// An item is one KV head, up to `span` consecutive tokens (their query heads of
// the group are its rows) and the keys that they see of one source: the shared
// prefix (all of the call's tokens together, whatever sequence they are of) or one
// sequence's own slots.  Its keys are cut into tiles of 128.  All items' tiles in a
// row (the prefix's by head and token group, then the own ones by head, sequence
// and token group) are dealt to the CTAs in equal runs, wherever items begin and
// end.  A tile counts a unit for each row tile that it meets (two take twice as
// long), and an item lead_units() more, for its queries, the start of its pipeline
// and its sums, so that a CTA with many short items has fewer tiles: whatever the
// lengths, all CTAs take about as long.  A CTA writes each of its items' unnormalised sum, maximum and sum of
// exponentials; a second kernel joins them row by row.  Partial sums are fp32.
#pragma once

#include <cuda.h>

#include "ecokv_decode.h"
#include "ecokv_internal.cuh"

namespace ecokv {

constexpr int kKeys = 128;        // keys a tile
constexpr int kTileRows = 128;    // most rows a partial sum of a continued item has
constexpr int kMaxGroup = 64;     // query heads a KV head
constexpr int kMaxAttendSms = 256;

struct AttendArgs {
  const void* q;
  void* out;
  float* lse;
  int64_t q_token, q_head, out_token, out_head;
  int tokens, batch, h_q, h_kv, g;
  ecokv_prefix prefix;    // rows 0: none
  ecokv_pages cache;
  int has_cache, page_shift, cap;  // cap: slots a sequence can have
  const int32_t* starts;
  const uint32_t* mask;  // a tree's: [tokens][words] of 32 bits, NULL: causal
  int words;
  int tpt;    // tokens a row tile holds
  int span;   // tokens an item holds (one or two row tiles)
  int groups, last;  // items that all tokens make, the last one's tokens
  int parts;  // row tiles that an item may have
  int P;      // CTAs
  int lead;   // see lead_units()
  int stall;  // fault injection: no tile ever comes
  float scale_log2;
  unsigned long long timeout_ns;
  // workspace
  float* first_o;   // [2 sources][tokens * h_q][d]: an item's sum from its first tile on
  float2* first_ml; //   maximum (log2 units) and sum
  float* next_o;    // [P][parts][kTileRows][d]: of an item that an earlier CTA began
  float2* next_ml;
  int* plan;        // see PLAN_*
  unsigned* status;
};

// What the attention kernel leaves for the joining one.
enum : int {
  PLAN_RUN = 0,       // units a CTA
  PLAN_PREFIX = 1,    // units of the prefix
  PLAN_OWN = 2,       // units of one head's own slots over all sequences
  PLAN_HEADS = 4      // [h_kv] first unit of each head's prefix, then [batch] first own unit of each sequence
};

struct Item {
  int source;         // 0 prefix, 1 own
  int head, seq;
  int tok0, ntok;     // tokens of the call
  int lim0, slope;    // token k of the item sees lim0 + k slope keys (at least 0); a tree's also
                      // those from lim0 on whose bit is set
  int vis;            // the most keys any of them sees
  int tile0, ntiles;  // this CTA's tiles of the item
  int row0;           // first row of the head's prefix (head_off)
};

__device__ __forceinline__ void note(const AttendArgs& a, unsigned code, unsigned detail) {
  if (atomicCAS(a.status, 0u, code) == 0u) a.status[1] = detail;
}

__host__ __device__ inline int div_up(int a, int b) { return (a + b - 1) / b; }
__host__ __device__ inline int tiles_of(int keys) { return (keys + kKeys - 1) >> 7; }  // (keys >= 0)
static_assert(kKeys == 128, "tiles_of");

// Tokens and slots of sequence b, clamped to what the buffers hold.
struct Seq {
  int start, T, L;
};
__device__ __forceinline__ Seq load_seq(const AttendArgs& a, int b, bool report) {
  Seq s;
  int s0 = b, s1 = b + 1;
  if (a.starts != nullptr) {
    s0 = a.starts[b];
    s1 = a.starts[b + 1];
  }
  const int len = a.cache.lengths[b];
  s.start = min(max(s0, 0), a.tokens);
  s.T = min(max(s1, s.start), a.tokens) - s.start;
  s.L = min(max(len, 0), a.cap);
  if (report && (s.L != len || s.start != s0 || s.start + s.T != s1)) note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)b);
  return s;
}
// Units of a tile of an item of so many tokens; those an item has before its first
// tile's (one row tile: 1, two: 4, their sums being up to 128 KB; at 1 for both 16
// sequences of 61 tokens over 6554 rows take 137 us, so 95; at 4 for both 61 single
// tokens of 32 heads over 1095 rows 67, so 42); all of an item's.
__host__ __device__ inline int tile_units(const AttendArgs& a, int ntok) { return ntok > a.tpt ? 2 : 1; }
__host__ __device__ inline int lead_units(const AttendArgs& a, int ntok) { return ntok > a.tpt ? 4 * a.lead : a.lead; }
__host__ __device__ inline int item_units(const AttendArgs& a, int tiles, int ntok) {
  return tiles > 0 ? tiles * tile_units(a, ntok) + lead_units(a, ntok) : 0;
}
// ... of all token groups of the prefix of one head (the last may be a shorter one).
__host__ __device__ inline int prefix_units(const AttendArgs& a, int tiles) {
  return (a.groups - 1) * item_units(a, tiles, a.span) + item_units(a, tiles, a.last);
}
// Keys that a sequence's item from its token i on sees at most, the item's units, and
// those of all its items from tokens below `until`.
__device__ __forceinline__ int seq_vis(const AttendArgs& a, const Seq& s, int i) {
  return a.mask != nullptr ? s.L : max(s.L - s.T + min(s.T, i + a.span), 0);
}
__device__ __forceinline__ int seq_item(const AttendArgs& a, const Seq& s, int i) {
  return item_units(a, tiles_of(seq_vis(a, s, i)), min(s.T - i, a.span));
}
__device__ __forceinline__ int seq_units(const AttendArgs& a, const Seq& s, int until) {
  int n = 0;
#pragma unroll 1
  for (int i = 0; i < until; i += a.span) n += seq_item(a, s, i);
  return n;
}
// Rows of head h's prefix.
__device__ __forceinline__ int prefix_rows(const AttendArgs& a, int h, int& row0, bool report) {
  row0 = 0;
  if (a.prefix.head_off == nullptr || a.prefix.rows == 0) return a.prefix.rows;
  const int o0 = a.prefix.head_off[h], o1 = a.prefix.head_off[h + 1];
  row0 = min(max(o0, 0), a.prefix.rows);
  const int n = min(max(o1, row0), a.prefix.rows) - row0;
  if (report && (row0 != o0 || row0 + n != o1)) note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)h);
  return n;
}

// A warp's walk over its CTA's run of units, item by item.  Every lane holds the
// same state but for the 32 sequences (or heads) at hand, one a lane.
struct Walk {
  int x, end;               // units of all items: next, one past the CTA's last
  int prefix_total, own;    // units of the prefix; of one head's own slots
  int lane;
  // the 32 sequences from b0 on: first unit of the first of them within a head
  int b0, base, head;
  Seq s;
  int w, upto;              // this lane's units, and those of lanes up to it

  static __device__ __forceinline__ int scan(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v = (int)((unsigned)v + (unsigned)u);  // (may wrap where begin() drops the sequences)
    }
    return v;
  }

  __device__ __forceinline__ void chunk(const AttendArgs& a, int from, bool report) {
    b0 = from;
    const int b = b0 + lane;
    s = Seq{0, 0, 0};
    w = 0;
    if (b < a.batch) {
      s = load_seq(a, b, report);
      w = seq_units(a, s, s.T);
    }
    upto = scan(w, lane);
  }

  // All of the warp's lanes.  The first CTA also leaves the plan.
  __device__ __forceinline__ void begin(const AttendArgs& a, int cta, int lane_) {
    lane = lane_;
    const bool lead = cta == 0;
    prefix_total = 0;
    if (a.prefix.rows > 0) {
      if (a.prefix.head_off == nullptr) {
        const int per = prefix_units(a, tiles_of(a.prefix.rows));
        prefix_total = a.h_kv * per;
        if (lead)
#pragma unroll 1
          for (int h = lane; h < a.h_kv; h += 32) a.plan[PLAN_HEADS + h] = h * per;
      } else {
#pragma unroll 1
        for (int h0 = 0; h0 < a.h_kv; h0 += 32) {
          int row0, n = 0;
          if (h0 + lane < a.h_kv) n = prefix_units(a, tiles_of(prefix_rows(a, h0 + lane, row0, lead)));
          const int up = scan(n, lane);
          if (lead && h0 + lane < a.h_kv) a.plan[PLAN_HEADS + h0 + lane] = prefix_total + up - n;
          prefix_total += __shfl_sync(0xffffffffu, up, 31);
        }
      }
    }
    own = 0;
    if (a.has_cache) {
      long long sum = 0;
#pragma unroll 1
      for (int c = 0; c < a.batch; c += 32) {
        chunk(a, c, lead);
        if (lead && c + lane < a.batch) a.plan[PLAN_HEADS + a.h_kv + c + lane] = (int)sum + upto - w;
        // (in 64 bits: starts that overlap may have every sequence hold all of the tokens)
        sum += __reduce_add_sync(0xffffffffu, (unsigned)w & 0xffffu) +
               ((long long)__reduce_add_sync(0xffffffffu, (unsigned)w >> 16) << 16);
      }
      // (valid starts stay below this, as the host has checked)
      if (sum * a.h_kv > 0x7fffffff - prefix_total) {
        if (lead && lane == 0) note(a, ECOKV_ERR_DEVICE_INDEX, (unsigned)a.batch);
        sum = 0;
      }
      own = (int)sum;
      if (a.batch > 32) chunk(a, 0, false);
    }
    base = 0;
    head = 0;
    const int total = prefix_total + a.h_kv * own;
    // (at least a tile's units: no CTA between the first and the last of an item is without a tile of it)
    // (in 32 bits without a sign: a run behind the last unit may begin past 31 bits)
    const int run = max((int)(((unsigned)total + (unsigned)a.P - 1u) / (unsigned)a.P), tile_units(a, a.span));
    if (lead && lane == 0) {
      a.plan[PLAN_RUN] = run;
      a.plan[PLAN_PREFIX] = prefix_total;
      a.plan[PLAN_OWN] = own;
    }
    x = (int)min((unsigned)cta * (unsigned)run, (unsigned)total);
    end = (int)min((unsigned)x + (unsigned)run, (unsigned)total);
  }

  // The next item (the same in every lane); false: none left.
  __device__ __forceinline__ bool next(const AttendArgs& a, Item& it) {
#pragma unroll 1
    while (x < end) {
      if (!at(a, it)) return false;
      if (it.ntiles > 0) return true;
    }
    return false;
  }
  // The part of an item from unit x on, which may be less than its first tile (ntiles <= 0).
  __device__ __forceinline__ bool at(const AttendArgs& a, Item& it) {
    int y, nt;  // place within the item; its tiles
    if (x < prefix_total) {
      int h, row0;
      if (a.prefix.head_off == nullptr) {
        const int per = prefix_units(a, tiles_of(a.prefix.rows));
        h = x / per;
        y = x - h * per;
        row0 = 0;
        it.vis = a.prefix.rows;
      } else {
        int at = 0;
        h = 0;
#pragma unroll 1
        for (int h0 = 0;; h0 += 32) {
          if (h0 >= a.h_kv) return false;  // (only when the offsets change under the kernel; so below)
          int n = 0, r0 = 0, rows = 0;
          if (h0 + lane < a.h_kv) {
            rows = prefix_rows(a, h0 + lane, r0, false);
            n = prefix_units(a, tiles_of(rows));
          }
          const int up = scan(n, lane), all = __shfl_sync(0xffffffffu, up, 31);
          if (x < at + all) {
            const int l = __ffs(__ballot_sync(0xffffffffu, x < at + up)) - 1;
            h = h0 + l;
            y = x - at - __shfl_sync(0xffffffffu, up - n, l);
            row0 = __shfl_sync(0xffffffffu, r0, l);
            it.vis = __shfl_sync(0xffffffffu, rows, l);
            break;
          }
          at += all;
        }
      }
      nt = tiles_of(it.vis);
      const int rg = y / item_units(a, nt, a.span);
      it.source = 0;
      it.head = h;
      it.seq = 0;
      it.tok0 = rg * a.span;
      it.ntok = min(a.span, a.tokens - it.tok0);
      it.lim0 = it.vis;
      it.slope = 0;
      y -= rg * item_units(a, nt, a.span);
      it.row0 = row0;
    } else {
      y = x - prefix_total;
      const int h = y / own;
      y -= h * own;
      if (h != head && b0 != 0) {
        base = 0;
        chunk(a, 0, false);
      }
      head = h;
      int all;
#pragma unroll 1
      while (y >= base + (all = __shfl_sync(0xffffffffu, upto, 31))) {
        base += all;
        if (b0 + 32 >= a.batch) return false;
        chunk(a, b0 + 32, false);
      }
      const int l = __ffs(__ballot_sync(0xffffffffu, y < base + upto)) - 1;
      y -= base + __shfl_sync(0xffffffffu, upto - w, l);
      Seq q;
      q.start = __shfl_sync(0xffffffffu, s.start, l);
      q.T = __shfl_sync(0xffffffffu, s.T, l);
      q.L = __shfl_sync(0xffffffffu, s.L, l);
      int i = 0, n;
#pragma unroll 1
      while (y >= (n = seq_item(a, q, i))) {
        y -= n;
        if ((i += a.span) >= q.T) return false;
      }
      it.source = 1;
      it.head = h;
      it.seq = b0 + l;
      it.tok0 = q.start + i;
      it.ntok = min(a.span, q.T - i);
      it.lim0 = a.mask != nullptr ? q.L - q.T : q.L - q.T + i + 1;
      it.slope = a.mask != nullptr ? 0 : 1;
      it.vis = seq_vis(a, q, i);
      it.row0 = 0;
      nt = tiles_of(it.vis);
    }
    // the tiles whose first unit lies within this CTA's part of the item, y .. z - 1
    const int u = tile_units(a, it.ntok), z = min(item_units(a, nt, it.ntok), y + end - x);
    const int lead = lead_units(a, it.ntok);
    it.tile0 = (max(y - lead, 0) + u - 1) >> (u - 1);  // (u: 1 or 2)
    it.ntiles = ((max(z - lead, 0) + u - 1) >> (u - 1)) - it.tile0;
    x += z - y;
    return z > y;  // (else nothing would move on)
  }
};

// Word w (32 drafts) of a token's row of the tree's mask; what lies before its sequence's
// drafts is seen.
__device__ __forceinline__ uint32_t tree_word(const AttendArgs& a, const uint32_t* row, int w) {
  return w < 0 ? ~0u : w < a.words ? row[w] : 0u;
}

// Where the sum of a row (token, query head) goes from its item's first CTA, and that
// of row `row` of row tile j of the item that CTA `cta` goes on with.
__device__ __forceinline__ size_t first_row(const AttendArgs& a, int source, int token, int hq) {
  return ((size_t)source * a.tokens + token) * a.h_q + hq;
}
__device__ __forceinline__ size_t next_row(const AttendArgs& a, int cta, int j, int row) {
  return ((size_t)cta * a.parts + j) * kTileRows + row;
}

// Argument checks of the decode step's entry points: addresses and strides (of elements
// of e bytes) in whole 16 bytes.
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline bool stride_ok(int64_t s, size_t e) { return ((uint64_t)s * e & 15u) == 0; }
// A tensor of bf16 rows of 128 for TMA, the axes after the first `strides` elements apart, in
// boxes of 64 columns with the 128-byte swizzle.
bool map_of(CUtensorMap* m, const void* base, int rank, const uint64_t* dims, const int64_t* strides,
            const uint32_t* box);
// CTAs of the persistent kernels: the current device's SMs.
int attend_sms();
ecokv_status check_pages(const ecokv_pages* c, int32_t batch, ecokv_dtype dt);
cudaError_t launch_attend_simt(const AttendArgs& a, ecokv_dtype dt, cudaStream_t st);
cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t st);
cudaError_t launch_attend_join(const AttendArgs& a, ecokv_dtype dt, cudaStream_t st);

}  // namespace ecokv
