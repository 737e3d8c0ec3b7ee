// ecokv_attend: argument checks, workspace, path choice, and the kernel that joins
// the partial sums.

#include <math.h>

#include "attend.cuh"
#include "ptx.cuh"

namespace ecokv {
namespace {

// kWarps warps a row (token, query head), kJoinWarps / kWarps rows a CTA: the row's
// partial sums, wherever the CTAs left them, weighted by 2^(their maximum - the
// largest).  Every warp finds the weights, 32 at a time, and sums those of its
// share; each lane has four columns.  What bounds it is the latency of its chain of
// loads, so a row with many parts has them read by four warps at once.
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

// Partial sums of one source that a row has: of CTAs c0 .. c0 + n / nj - 1.
struct Parts {
  int c0, n, nj, j0;
  size_t first;   // row of the first CTA's
  int row;        // row within a continued item
};

// (unit: the item's first; nt: its tiles)
__device__ __forceinline__ Parts find_parts(const AttendArgs& a, int source, int unit, int nt, int run, int k, int ntok,
                                            int token, int hq) {
  Parts p{0, 0, 1, 0, 0, 0};
  if (nt <= 0) return p;
  unit += lead_units(a, ntok);
  p.c0 = unit / run;
  const int ctas = (unit + (nt - 1) * tile_units(a, ntok)) / run - p.c0 + 1;
  if (ntok > a.tpt) p.j0 = k / a.tpt;  // two row tiles: the row is in one of them
  else p.nj = a.parts;
  p.n = ctas * p.nj;
  p.first = first_row(a, source, p.j0, token, hq);
  p.row = (k % a.tpt) * a.g + hq % a.g;
  return p;
}

__device__ __forceinline__ const float* part(const AttendArgs& a, const Parts& p, int e, float2& ml) {
  const int c = e / p.nj, j = e - c * p.nj;
  if (c == 0) {
    const size_t at = p.first + (size_t)j * a.tokens * a.h_q;
    ml = a.first_ml[at];
    return a.first_o + at * kD;
  }
  const size_t at = next_row(a, p.c0 + c, p.j0 + j, p.row);
  ml = a.next_ml[at];
  return a.next_o + at * kD;
}

template <typename T, int kWarps>
__global__ void __launch_bounds__(32 * kJoinWarps) attend_join_kernel(const __grid_constant__ AttendArgs a) {
  __shared__ float4 part_acc[kJoinWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp % kWarps;
  const long long id = (long long)blockIdx.x * (kJoinWarps / kWarps) + warp / kWarps;
  if (id >= (long long)a.tokens * a.h_q) return;  // (with kWarps = kJoinWarps the whole CTA)
  const int token = (int)(id / a.h_q), hq = (int)(id - (long long)token * a.h_q), h = hq / a.g;
  Parts src[2] = {{0, 0, 1, 0, 0, 0}, {0, 0, 1, 0, 0, 0}};
  const int run = a.plan[PLAN_RUN], prefix_total = a.plan[PLAN_PREFIX], own = a.plan[PLAN_OWN];
  if (a.prefix.rows > 0) {
    int row0;
    const int nt = div_up(prefix_rows(a, h, row0, false), kKeys), rg = token / a.span;
    src[0] = find_parts(a, 0, a.plan[PLAN_HEADS + h] + rg * item_units(a, nt, a.span), nt, run, token - rg * a.span,
                        min(a.span, a.tokens - rg * a.span), token, hq);
  }
  if (a.has_cache) {
    int b = token;
    if (a.starts != nullptr) {
      b = 0;
      for (int j = lane; j < a.batch; j += 32) b += a.starts[1 + j] <= token ? 1 : 0;
      b = min((int)__reduce_add_sync(0xffffffffu, (unsigned)b), a.batch - 1);
    }
    const int first = a.plan[PLAN_HEADS + a.h_kv + b];
    const Seq s = load_seq(a, b, false);
    const int i = token - s.start;
    if (i >= 0 && i < s.T && own > 0) {
      const int rg = i / a.span;
      src[1] = find_parts(a, 1, prefix_total + h * own + first + seq_units(a, s, rg),
                          div_up(seq_vis(a, s, rg), kKeys), run, i - rg * a.span, min(a.span, s.T - rg * a.span),
                          token, hq);
    }
  }
  // the parts of both sources in one row: entry e < src[0].n is the prefix's
  const int n = src[0].n + src[1].n;
  float M = -INFINITY, M0 = -INFINITY, l0 = 0.f;
  const float* o0 = nullptr;
  for (int e = lane; e < n; e += 32) {
    float2 ml;
    const float* o = e < src[0].n ? part(a, src[0], e, ml) : part(a, src[1], e - src[0].n, ml);
    if (e == lane) {
      o0 = o;
      M0 = ml.x;
      l0 = ml.y;
    }
    M = fmaxf(M, ml.x);
  }
  M = ptx::redux_max(M);
  const float ref = M == -INFINITY ? 0.f : M;
  float L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int e0 = 0; e0 < n; e0 += 32) {
    if (e0 > 0 && e0 + lane < n) {
      float2 ml;
      const int e = e0 + lane;
      o0 = e < src[0].n ? part(a, src[0], e, ml) : part(a, src[1], e - src[0].n, ml);
      M0 = ml.x;
      l0 = ml.y;
    }
    const float w = e0 + lane < n ? ptx::ex2(M0 - ref) : 0.f;
    L = fmaf(w, w > 0.f ? l0 : 0.f, L);
    const int k1 = min(32, n - e0);
#pragma unroll 8
    for (int k = mine; k < k1; k += kWarps) {
      const float wk = __shfl_sync(0xffffffffu, w, k);
      const float* ok = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, (unsigned long long)o0, k));
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (wk > 0.f) v = *reinterpret_cast<const float4*>(ok + 4 * lane);  // (a part that saw no key is not written)
      acc.x = fmaf(wk, v.x, acc.x);
      acc.y = fmaf(wk, v.y, acc.y);
      acc.z = fmaf(wk, v.z, acc.z);
      acc.w = fmaf(wk, v.w, acc.w);
    }
  }
  if constexpr (kWarps > 1) {
    part_acc[warp][lane] = acc;
    __syncthreads();
    if (mine != 0) return;
#pragma unroll
    for (int k = 1; k < kWarps; ++k) {
      const float4 v = part_acc[warp + k][lane];
      acc.x += v.x;
      acc.y += v.y;
      acc.z += v.z;
      acc.w += v.w;
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) L += __shfl_xor_sync(0xffffffffu, L, d);
  const float inv = L > 0.f ? 1.f / L : 0.f;
  acc.x *= inv;
  acc.y *= inv;
  acc.z *= inv;
  acc.w *= inv;
  store4(static_cast<T*>(a.out) + (int64_t)token * a.out_token + (int64_t)hq * a.out_head + 4 * lane, acc);
  if (a.lse != nullptr && lane == 0)
    a.lse[(int64_t)token * a.h_q + hq] = L > 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool stride_ok(int64_t s, size_t e) { return ((uint64_t)s * e & 15u) == 0; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct AttendLayout {
  size_t plan, first_ml, first_o, next_ml, next_o, total;
};
AttendLayout attend_layout(int32_t tokens, int32_t batch, int32_t h_q, int32_t h_kv, int parts) {
  AttendLayout L{};
  const size_t first = 2ull * parts * tokens * h_q, next = (size_t)kMaxAttendSms * parts * kTileRows;
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

int attend_sms() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
    n = 152;
  return n < kMaxAttendSms ? n : kMaxAttendSms;
}

template <typename T>
cudaError_t launch_join(const AttendArgs& a, cudaStream_t st) {
  const long long rows = (long long)a.tokens * a.h_q;
  // four warps a row while the rows are few (and so have many parts each)
  const bool wide = rows <= 2048;
  const unsigned grid = (unsigned)(wide ? rows : (rows + kJoinWarps - 1) / kJoinWarps);
  if (wide) attend_join_kernel<T, kJoinWarps><<<grid, 32 * kJoinWarps, 0, st>>>(a);
  else attend_join_kernel<T, 1><<<grid, 32 * kJoinWarps, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace

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

ecokv_status ecokv_attend(const ecokv_attend_params* p, ecokv_dtype dtype, const void* q, const ecokv_prefix* prefix,
                          const ecokv_pages* cache, const int32_t* starts, void* out, float* lse, void* ws,
                          size_t ws_bytes, void* stream) {
  if (p == nullptr || !sizes_ok(p->tokens, p->batch, p->h_q, p->h_kv) || p->d < 1) return ECOKV_ERR_INVALID_ARG;
  if (dtype != ECOKV_F32 && dtype != ECOKV_BF16) return ECOKV_ERR_INVALID_ARG;
  const size_t e = dtype == ECOKV_F32 ? 4 : 2;
  if ((p->flags & ~(ECOKV_FLAG_FORCE_SIMT | ECOKV_FLAG_TEST_STALL)) != 0u || !isfinite(p->scale))
    return ECOKV_ERR_INVALID_ARG;
  const bool tc = dtype == ECOKV_BF16 && (p->flags & ECOKV_FLAG_FORCE_SIMT) == 0u;
  if ((p->flags & ECOKV_FLAG_TEST_STALL) != 0u && !tc) return ECOKV_ERR_UNSUPPORTED;  // the waits are on that path
  if (p->d != kD || p->h_q / p->h_kv > kMaxGroup) return ECOKV_ERR_UNSUPPORTED;
  if (!q || !out || !aligned16(q) || !aligned16(out) || ((uintptr_t)lse & 3u)) return ECOKV_ERR_INVALID_ARG;
  if (p->q_token < 0 || p->q_head < 0 || p->out_token < 0 || p->out_head < 0 || !stride_ok(p->q_token, e) ||
      !stride_ok(p->q_head, e) || !stride_ok(p->out_token, e) || !stride_ok(p->out_head, e))
    return ECOKV_ERR_INVALID_ARG;
  AttendArgs a{};
  if (prefix != nullptr && prefix->rows != 0) {
    if (prefix->rows < 0 || !prefix->k || !prefix->v || !aligned16(prefix->k) || !aligned16(prefix->v) ||
        ((uintptr_t)prefix->head_off & 3u) || prefix->row_stride <= 0 || !stride_ok(prefix->row_stride, e) ||
        (!prefix->head_off && (prefix->head_stride < 0 || !stride_ok(prefix->head_stride, e))))
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
  if (ws == nullptr || !aligned16(ws) || ws_bytes < attend_layout(p->tokens, p->batch, p->h_q, p->h_kv, 2).total)
    return ECOKV_ERR_WORKSPACE;
  if (p->tokens == 0) return ECOKV_OK;
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
  a.span = tc ? 2 * a.tpt : a.tpt;
  a.parts = tc ? 2 : 1;
  a.lead = tc ? 1 : 0;
  a.stall = (p->flags & ECOKV_FLAG_TEST_STALL) ? 1 : 0;
  a.P = attend_sms();
  const double scale = p->scale > 0.f ? (double)p->scale : 1.0 / sqrt((double)kD);
  a.scale_log2 = (float)(1.4426950408889634 * scale);
  a.timeout_ns = (p->timeout_us ? (unsigned long long)p->timeout_us : 2000000ull) * 1000ull;
  // units of every item, counted in 32 bits by the kernels
  const long long groups = (a.tokens + a.span - 1) / a.span;
  const long long of_cap = item_units(a, (a.cap + kKeys - 1) / kKeys, a.span),
                  of_prefix = item_units(a, (a.prefix.rows + kKeys - 1) / kKeys, a.span);
  const long long units = a.h_kv * (groups * of_prefix + (groups + a.batch) * of_cap);
  if (units > 0x7fffffff || groups * of_cap > (1 << 25)) return ECOKV_ERR_UNSUPPORTED;
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

}  // extern "C"
