// ecokv_attend: argument checks, workspace, path choice, and the kernel that joins
// the partial sums.

#include <math.h>

#include <atomic>

#include "attend.cuh"
#include "decode_ptx.cuh"
#include "tc_tile.cuh"

namespace ecokv {
namespace {

// A row's (token, query head) partial sums, wherever the CTAs left them, weighted by
// 2^(their maximum - the largest).  What bounds this is the latency of its chain of
// loads.  With few rows a CTA takes one, its warps a share of the parts each, and the
// sums are loaded beside the weights that may turn out to be zero; with many rows
// a warp takes rows of one token and KV head, whose parts lie side by side and are
// looked up once.
// Each lane has four columns.
constexpr int kJoinWarps = 4;

template <typename T>
__device__ __forceinline__ void store4(T* p, float4 v);
template <>
__device__ __forceinline__ void store4<float>(float* p, float4 v) {
  *reinterpret_cast<float4*>(p) = v;
}
template <>
__device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16* p, float4 v) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) =
      make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

// Partial sums of one source that a row has: one of each of n CTAs from c0 on.
struct Parts {
  int c0, n, tile;
  size_t first;   // row of the first CTA's
  int row;        // row of row tile `tile` of a continued item
};

// (unit: the item's first; nt: its tiles)
__device__ __forceinline__ Parts find_parts(const AttendArgs& a, int source, int unit, int nt, int run, int k, int ntok,
                                            int token, int hq) {
  Parts p{0, 0, 0, 0, 0};
  if (nt <= 0) return p;
  unit += lead_units(a, ntok);
  p.c0 = unit / run;
  p.n = (unit + (nt - 1) * tile_units(a, ntok)) / run - p.c0 + 1;
  p.tile = k >= a.tpt ? 1 : 0;
  p.first = first_row(a, source, token, hq);
  p.row = (k - p.tile * a.tpt) * a.g + hq % a.g;
  return p;
}

__device__ __forceinline__ const float* part(const AttendArgs& a, const Parts& p, int e, float2& ml) {
  if (e == 0) {
    ml = a.first_ml[p.first];
    return a.first_o + p.first * kD;
  }
  const size_t at = next_row(a, p.c0 + e, p.tile, p.row);
  ml = a.next_ml[at];
  return a.next_o + at * kD;
}

// The parts of both sources of a row in one list: entry e < src[0].n is the prefix's.
struct PartList {
  Parts src[2];
  int n;
  // (row r of the token's rows of the KV head, of which row 0 was looked up)
  __device__ __forceinline__ const float* at(const AttendArgs& a, int e, int r, float2& ml) const {
    const bool second = e >= src[0].n;
    Parts p = second ? src[1] : src[0];
    p.first += r;
    p.row += r;
    return part(a, p, second ? e - src[0].n : e, ml);
  }
};

__device__ __forceinline__ PartList list_parts(const AttendArgs& a, int token, int h, int lane) {
  PartList l{};
  int b = token;
  if (a.has_cache && a.starts != nullptr) {
    b = 0;
    for (int j = lane; j < a.batch; j += 32) b += a.starts[1 + j] <= token ? 1 : 0;
    b = min((int)__reduce_add_sync(0xffffffffu, (unsigned)b), a.batch - 1);
  }
  const int4 head = *reinterpret_cast<const int4*>(a.plan);
  const int run = head.x, prefix_total = head.y, own = head.z;
  if (a.prefix.rows > 0) {
    int row0;
    const int first = a.plan[PLAN_HEADS + h];
    const int nt = tiles_of(prefix_rows(a, h, row0, false)), rg = token / a.span;
    l.src[0] = find_parts(a, 0, first + rg * item_units(a, nt, a.span), nt, run, token - rg * a.span,
                          min(a.span, a.tokens - rg * a.span), token, h * a.g);
  }
  if (a.has_cache) {
    const int first = a.plan[PLAN_HEADS + a.h_kv + b];
    const Seq s = load_seq(a, b, false);
    const int i = token - s.start;
    if (i >= 0 && i < s.T && own > 0) {
      const int i0 = i / a.span * a.span;  // its item's first token
      l.src[1] = find_parts(a, 1, prefix_total + h * own + first + seq_units(a, s, i0), tiles_of(seq_vis(a, s, i0)),
                            run, i - i0, min(a.span, s.T - i0), token, h * a.g);
    }
  }
  l.n = l.src[0].n + l.src[1].n;
  return l;
}

// acc += w v, v = 0 where w is (a part that saw no key is not written).
__device__ __forceinline__ void add_part(float4& acc, float w, float4 v) {
  const bool any = w > 0.f;
  acc.x = fmaf(w, any ? v.x : 0.f, acc.x);
  acc.y = fmaf(w, any ? v.y : 0.f, acc.y);
  acc.z = fmaf(w, any ? v.z : 0.f, acc.z);
  acc.w = fmaf(w, any ? v.w : 0.f, acc.w);
}

// The weight of this lane's next part: the largest maximum M, the lane's share L of the
// sum and the output so far follow.
__device__ __forceinline__ float next_weight(float& M, float& L, float4& acc, float2 ml) {
  const float Mn = fmaxf(M, ptx::redux_max(ml.x)), ref = Mn == -INFINITY ? 0.f : Mn;
  const float c = ptx::ex2(M - ref), w = ptx::ex2(ml.x - ref);
  M = Mn;
  L = fmaf(L, c, w > 0.f ? w * ml.y : 0.f);
  acc.x *= c;
  acc.y *= c;
  acc.z *= c;
  acc.w *= c;
  return w;
}

template <typename T>
__device__ __forceinline__ void store_row(const AttendArgs& a, int token, int hq, int lane, float4 acc, float M,
                                          float L) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) L += __shfl_xor_sync(0xffffffffu, L, d);
  const float inv = L > 0.f ? 1.f / L : 0.f;
  acc.x *= inv;
  acc.y *= inv;
  acc.z *= inv;
  acc.w *= inv;
  store4(static_cast<T*>(a.out) + (int64_t)token * a.out_token + (int64_t)hq * a.out_head + 4 * lane, acc);
  if (a.lse != nullptr && lane == 0) {
    // (L is at least 1/2 unless it is 0; infinite or NaN only where an input was)
    const float x = L < INFINITY ? log2_sum(M, L) : L;
    a.lse[(int64_t)token * a.h_q + hq] = L == 0.f ? -INFINITY : x * 0.6931471805599453f;
  }
}

constexpr int kAhead = 32 / kJoinWarps;  // sums whose loads a warp has in flight

// One warp `per` rows of a (token, KV head).
template <typename T>
__global__ void __launch_bounds__(32 * kJoinWarps, 8)
    attend_join_heads_kernel(const __grid_constant__ AttendArgs a, int per, int split) {
  // (the next call's first kernel is scheduled behind this one)
  ptx::grid_trigger();
  ptx::grid_wait();
  const int lane = threadIdx.x & 31;
  const long long id = (long long)blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
  if (id >= (long long)a.tokens * a.h_kv * split) return;
  const long long unit = id / split;
  const int token = (int)(unit / a.h_kv), h = (int)(unit - (long long)token * a.h_kv);
  const int r0 = (int)(id - unit * split) * per, r1 = min(r0 + per, a.g);
  const PartList l = list_parts(a, token, h, lane);
  // (a row's first 32 parts are looked up while the row before it is summed)
  float2 ml_next = make_float2(-INFINITY, 0.f);
  const float* o_next = nullptr;
#pragma unroll 1
  for (int r = r0 - 1; r < r1; ++r) {
    const float* o = o_next;
    float2 ml = ml_next;
    if (lane < l.n && r + 1 < r1) o_next = l.at(a, lane, r + 1, ml_next);
    if (r < r0) continue;
    float M = -INFINITY, L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int e0 = 0; e0 < l.n; e0 += 32) {
      if (e0 > 0) {
        ml = make_float2(-INFINITY, 0.f);
        if (e0 + lane < l.n) o = l.at(a, e0 + lane, r, ml);
      }
      const float w = next_weight(M, L, acc, ml);
      const int n = min(32, l.n - e0);
      // (in one order; past two sums the loads of four at once: 768 drafts of 28 heads 68.3 us,
      // 70.5 one after another.  Eight CTAs an SM, 64 registers a thread and 28 bytes of it
      // spilled: without that bound 3000 tokens of 32 heads, of few sums a row, take 167 us and
      // not 162.5.)
      if (n <= 2) {
#pragma unroll 2
        for (int k = 0; k < n; ++k) {
          const float* ok = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, (unsigned long long)o, k));
          add_part(acc, __shfl_sync(0xffffffffu, w, k), *reinterpret_cast<const float4*>(ok + 4 * lane));
        }
        continue;
      }
#pragma unroll 1
      for (int k0 = 0; k0 < n; k0 += 4) {
        float4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float* ok = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, (unsigned long long)o, k0 + k));
          v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (k0 + k < n) v[k] = *reinterpret_cast<const float4*>(ok + 4 * lane);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float wk = __shfl_sync(0xffffffffu, w, k0 + k);
          if (k0 + k < n) add_part(acc, wk, v[k]);
        }
      }
    }
    store_row<T>(a, token, h * a.g + r, lane, acc, M, L);
  }
}

// One CTA a row.
template <typename T>
__global__ void __launch_bounds__(32 * kJoinWarps) attend_join_row_kernel(const __grid_constant__ AttendArgs a) {
  __shared__ float4 sums[kJoinWarps][32];
  ptx::grid_trigger();
  ptx::grid_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int token = blockIdx.x / a.h_q, hq = blockIdx.x - token * a.h_q, h = hq / a.g, r = hq - h * a.g;
  const PartList l = list_parts(a, token, h, lane);
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  // (32 parts are looked up while those before them are summed)
  float2 ml_next = make_float2(-INFINITY, 0.f);
  const float* o_next = nullptr;
#pragma unroll 1
  for (int e0 = -32; e0 < l.n; e0 += 32) {
    const float* o = o_next;
    const float2 ml = ml_next;
    ml_next = make_float2(-INFINITY, 0.f);
    if (e0 + 32 + lane < l.n) o_next = l.at(a, e0 + 32 + lane, r, ml_next);
    if (e0 < 0) continue;
    float4 v[kAhead];  // this warp's sums of these 32
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = k * kJoinWarps + warp;
      const float* ok = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, (unsigned long long)o, e));
      v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (e0 + e < l.n) v[k] = *reinterpret_cast<const float4*>(ok + 4 * lane);
    }
    const float w = next_weight(M, L, acc, ml);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) add_part(acc, __shfl_sync(0xffffffffu, w, k * kJoinWarps + warp), v[k]);
  }
  sums[warp][lane] = acc;
  __syncthreads();
  if (warp != 0) return;
#pragma unroll
  for (int k = 1; k < kJoinWarps; ++k) {
    const float4 x = sums[k][lane];
    acc.x += x.x;
    acc.y += x.y;
    acc.z += x.z;
    acc.w += x.w;
  }
  store_row<T>(a, token, hq, lane, acc, M, L);
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct AttendLayout {
  size_t plan, first_ml, first_o, next_ml, next_o, total;
};
AttendLayout attend_layout(int32_t tokens, int32_t batch, int32_t h_q, int32_t h_kv, int parts) {
  AttendLayout L{};
  const size_t first = 2ull * tokens * h_q, next = (size_t)kMaxAttendSms * parts * kTileRows;
  size_t off = 256;  // the status word
  L.plan = off;
  off += align256(((size_t)PLAN_HEADS + h_kv + batch) * 4);
  L.first_ml = off;
  off += align256(first * sizeof(float2));
  L.next_ml = off;
  off += align256(next * sizeof(float2));
  L.first_o = off;
  off += align256(first * kD * sizeof(float));
  L.next_o = off;
  off += align256(next * kD * sizeof(float));
  L.total = off;
  return L;
}
bool sizes_ok(int32_t tokens, int32_t batch, int32_t h_q, int32_t h_kv) {
  return tokens >= 0 && batch >= 1 && h_q >= 1 && h_kv >= 1 && h_q % h_kv == 0 && h_q <= (1 << 16);
}

template <typename T>
cudaError_t launch_join(const AttendArgs& a, cudaStream_t st) {
  const long long rows = (long long)a.tokens * a.h_q;
  // one CTA a row while all of them are resident (152 SMs of 8; the whole call at 1024
  // rows, 32 tokens over 131072 keys: 93.8 us so, 97.5 by warps; at 1792, 64 sequences of
  // up to 4096 slots: 62.4 and 60.5), past that as many rows a warp as leave 20 warps an SM
  // (3696 rows, 132 single tokens over 3277: 32.6 us, 34.2 at 10)
  if (rows <= 152 * 8) return launch_behind(attend_join_row_kernel<T>, (unsigned)rows, 32 * kJoinWarps, 0, st, a);
  const long long want = rows / (152 * 20);
  const int per = (int)(want < 1 ? 1 : want > a.g ? a.g : want), split = div_up(a.g, per);
  const long long warps = (long long)a.tokens * a.h_kv * split;
  return launch_behind(attend_join_heads_kernel<T>, (unsigned)((warps + kJoinWarps - 1) / kJoinWarps),
                       32 * kJoinWarps, 0, st, a, per, split);
}

}  // namespace

// (cached per device; a racing thread repeats the query)
int attend_sms() {
  static std::atomic<int> cached[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 152;
  if ((n = cached[dev].load()) == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 152;
    cached[dev].store(n);
  }
  return n < kMaxAttendSms ? n : kMaxAttendSms;
}

ecokv_status check_pages(const ecokv_pages* c, int32_t batch, ecokv_dtype dt) {
  if (c == nullptr || batch < 1) return ECOKV_ERR_INVALID_ARG;
  const size_t e = dt == ECOKV_F32 ? 4 : 2;
  if (!c->k || !c->v || !c->table || !c->lengths) return ECOKV_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || ((uintptr_t)c->table & 3u) || ((uintptr_t)c->lengths & 3u))
    return ECOKV_ERR_INVALID_ARG;
  if (c->page_stride <= 0 || c->head_stride <= 0 || c->slot_stride <= 0 || !stride_ok(c->page_stride, e) ||
      !stride_ok(c->head_stride, e) || !stride_ok(c->slot_stride, e))
    return ECOKV_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->table_stride < 1) return ECOKV_ERR_INVALID_ARG;
  if (c->page_size < 8 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0)
    return ECOKV_ERR_INVALID_ARG;
  if ((long long)c->page_size * c->table_stride > kMaxN) return ECOKV_ERR_UNSUPPORTED;
  return ECOKV_OK;
}

cudaError_t launch_attend_join(const AttendArgs& a, ecokv_dtype dt, cudaStream_t st) {
  return dt == ECOKV_F32 ? launch_join<float>(a, st) : launch_join<__nv_bfloat16>(a, st);
}

}  // namespace ecokv

using namespace ecokv;

extern "C" {

size_t ecokv_attend_workspace_size(int32_t tokens, int32_t batch, int32_t h_q, int32_t h_kv, ecokv_dtype dtype) {
  if (!sizes_ok(tokens, batch, h_q, h_kv) || (dtype != ECOKV_F32 && dtype != ECOKV_BF16)) return 0;
  return attend_layout(tokens, batch, h_q, h_kv, 2).total;
}

}  // extern "C"

static ecokv_status attend(const ecokv_attend_params* p, ecokv_dtype dtype, const void* q, const ecokv_prefix* prefix,
                           const ecokv_pages* cache, const int32_t* starts, const uint64_t* mask, int32_t words,
                           void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (p == nullptr || !sizes_ok(p->tokens, p->batch, p->h_q, p->h_kv) || p->d < 1) return ECOKV_ERR_INVALID_ARG;
  if (dtype != ECOKV_F32 && dtype != ECOKV_BF16) return ECOKV_ERR_INVALID_ARG;
  const size_t e = dtype == ECOKV_F32 ? 4 : 2;
  if ((p->flags & ~(ECOKV_FLAG_FORCE_SIMT | ECOKV_FLAG_TEST_STALL)) != 0u || !isfinite(p->scale))
    return ECOKV_ERR_INVALID_ARG;
  const bool tc = dtype == ECOKV_BF16 && (p->flags & ECOKV_FLAG_FORCE_SIMT) == 0u;
  if ((p->flags & ECOKV_FLAG_TEST_STALL) != 0u && !tc) return ECOKV_ERR_UNSUPPORTED;  // the waits are on that path
  if (p->d != kD || p->h_q / p->h_kv > kMaxGroup) return ECOKV_ERR_UNSUPPORTED;
  if (p->tokens == 0) return ECOKV_OK;  // (tensors of no rows may have no address)
  if (!q || !out || !aligned16(q) || !aligned16(out) || ((uintptr_t)lse & 3u)) return ECOKV_ERR_INVALID_ARG;
  if (p->q_token <= 0 || p->q_head <= 0 || p->out_token <= 0 || p->out_head <= 0 || !stride_ok(p->q_token, e) ||
      !stride_ok(p->q_head, e) || !stride_ok(p->out_token, e) || !stride_ok(p->out_head, e))
    return ECOKV_ERR_INVALID_ARG;
  AttendArgs a{};
  if (prefix != nullptr && prefix->rows != 0) {
    if (prefix->rows < 0 || !prefix->k || !prefix->v || !aligned16(prefix->k) || !aligned16(prefix->v) ||
        ((uintptr_t)prefix->head_off & 3u) || prefix->row_stride <= 0 || !stride_ok(prefix->row_stride, e) ||
        (!prefix->head_off && (prefix->head_stride <= 0 || !stride_ok(prefix->head_stride, e))))
      return ECOKV_ERR_INVALID_ARG;
    if (prefix->rows > kMaxN) return ECOKV_ERR_UNSUPPORTED;
    a.prefix = *prefix;
  }
  if (cache != nullptr) {
    const ecokv_status st = check_pages(cache, p->batch, dtype);
    if (st != ECOKV_OK) return st;
    if ((uintptr_t)starts & 3u || (starts == nullptr && p->tokens != p->batch)) return ECOKV_ERR_INVALID_ARG;
    a.cache = *cache;
    a.has_cache = 1;
    a.page_shift = __builtin_ctz((unsigned)cache->page_size);
    a.cap = cache->page_size * cache->table_stride;
    a.starts = starts;
  }
  a.mask = reinterpret_cast<const uint32_t*>(mask);  // (both machines' words are little-endian)
  a.words = 2 * words;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.q_token = p->q_token;
  a.q_head = p->q_head;
  a.out_token = p->out_token;
  a.out_head = p->out_head;
  a.tokens = p->tokens;
  a.batch = p->batch;
  a.h_q = p->h_q;
  a.h_kv = p->h_kv;
  a.g = p->h_q / p->h_kv;
  a.tpt = (tc ? kTileRows : 64) / a.g;
  // A tree on CUDA cores: row tiles of 16 where even those are few, one or two a CTA (two take the time
  // of one of 64, whose rows cost less each: 8 trees of up to 13 drafts, 8 heads, 128 rows before
  // them and up to 200 slots 16.5 us, 24.4 in 64s; one of 64 drafts over 4000 slots 68.6 and 41.6.
  // Of 70 batches of 1 to 32 trees this takes 1.02 times the better of the two, 64 rows
  // always 1.05, 16 always 1.45).  A table with room for more than is in use counts in full, and
  // a call is then cut in 64s.
  if (!tc && mask != nullptr && a.g <= 16) {
    const int few = 16 / a.g;
    const double groups = (a.tokens - 1) / few + 1, each = (a.tokens - 1) / a.batch / few + 1;
    if (a.h_kv * (groups * tiles_of(a.prefix.rows) + a.batch * each * tiles_of(a.cap)) <= 1.5 * attend_sms())
      a.tpt = few;
  }
  a.span = tc ? 2 * a.tpt : a.tpt;
  a.parts = tc ? 2 : 1;
  a.lead = tc ? 1 : 0;
  a.stall = (p->flags & ECOKV_FLAG_TEST_STALL) ? 1 : 0;
  const double scale = p->scale > 0.f ? (double)p->scale : 1.0 / sqrt((double)kD);
  a.scale_log2 = (float)(1.4426950408889634 * scale);
  a.timeout_ns = (p->timeout_us ? (unsigned long long)p->timeout_us : 2000000ull) * 1000ull;
  // Units of every item, counted in 32 bits by the kernels: as many as there can be of the
  // sequences' slots.  (A sequence's tokens make an item more than their share of the groups.)
  a.groups = (a.tokens - 1) / a.span + 1;
  a.last = a.tokens - (a.groups - 1) * a.span;
  const double groups = a.groups, of_cap = item_units(a, tiles_of(a.cap), a.span);
  const double of_prefix = item_units(a, tiles_of(a.prefix.rows), a.span);
  if (a.h_kv * (groups * of_prefix + (groups + a.batch) * of_cap) > 0x7fffffff) return ECOKV_ERR_UNSUPPORTED;
  if (ws == nullptr || !aligned16(ws) || ws_bytes < attend_layout(p->tokens, p->batch, p->h_q, p->h_kv, 2).total)
    return ECOKV_ERR_WORKSPACE;
  a.P = attend_sms();
  char* w = static_cast<char*>(ws);
  const AttendLayout L = attend_layout(a.tokens, a.batch, a.h_q, a.h_kv, a.parts);
  a.status = reinterpret_cast<unsigned*>(w);
  a.plan = reinterpret_cast<int*>(w + L.plan);
  a.first_ml = reinterpret_cast<float2*>(w + L.first_ml);
  a.next_ml = reinterpret_cast<float2*>(w + L.next_ml);
  a.first_o = reinterpret_cast<float*>(w + L.first_o);
  a.next_o = reinterpret_cast<float*>(w + L.next_o);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((tc ? launch_attend_tc(a, s) : launch_attend_simt(a, dtype, s)) != cudaSuccess) return ECOKV_ERR_CUDA;
  return launch_attend_join(a, dtype, s) == cudaSuccess ? ECOKV_OK : ECOKV_ERR_CUDA;
}

extern "C" {

ecokv_status ecokv_attend(const ecokv_attend_params* p, ecokv_dtype dtype, const void* q, const ecokv_prefix* prefix,
                          const ecokv_pages* cache, const int32_t* starts, void* out, float* lse, void* ws,
                          size_t ws_bytes, void* stream) {
  return attend(p, dtype, q, prefix, cache, starts, nullptr, 0, out, lse, ws, ws_bytes, stream);
}

ecokv_status ecokv_attend_tree(const ecokv_attend_params* p, ecokv_dtype dtype, const void* q,
                               const ecokv_prefix* prefix, const ecokv_pages* cache, const int32_t* starts,
                               const uint64_t* mask, int32_t words, void* out, float* lse, void* ws, size_t ws_bytes,
                               void* stream) {
  if (words < 1) return ECOKV_ERR_INVALID_ARG;
  if (words > 64) return ECOKV_ERR_UNSUPPORTED;
  if (p != nullptr && p->tokens != 0 && (cache == nullptr || mask == nullptr || ((uintptr_t)mask & 7u)))
    return ECOKV_ERR_INVALID_ARG;
  return attend(p, dtype, q, prefix, cache, starts, mask, words, out, lse, ws, ws_bytes, stream);
}

}  // extern "C"
