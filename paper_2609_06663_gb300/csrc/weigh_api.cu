// ecokv_weigh: argument checks, workspace, path choice, and the kernel that adds what
// further CTAs of an item have left.

#include <math.h>

#include "decode_ptx.cuh"
#include "weigh.cuh"

namespace ecokv {
namespace {

// Block c: the item that CTA c goes on with, if it is the first one that does; the sums of
// those behind it follow in their order.
__global__ void __launch_bounds__(kWeighSpan) weigh_join_kernel(const __grid_constant__ WeighArgs w) {
  ptx::grid_trigger();
  ptx::grid_wait();
  const int c = blockIdx.x;
  const WeighItem it = w.next_item[c];
  if (it.tile0 == 0) return;
  auto same = [&](const WeighItem& o) {
    return o.tile0 != 0 && o.source == it.source && o.head == it.head && o.seq == it.seq && o.key0 == it.key0;
  };
  if (c > 0 && same(w.next_item[c - 1])) return;
  const int k = threadIdx.x;
  // (the last CTA of the item, 32 looked at at once, then independent loads)
  int last = c;
  for (int o = c + 1; o < w.a.P; o += 32) {
    const int i = o + (k & 31);
    const unsigned m = __ballot_sync(0xffffffffu, i < w.a.P && same(w.next_item[min(i, w.a.P - 1)]));
    last += m == ~0u ? 32 : __ffs(~m) - 1;
    if (m != ~0u) break;
  }
  float sum = 0.f;
#pragma unroll 8
  for (int o = c; o <= last; ++o) sum += w.next[(int64_t)o * kWeighSpan + k];
  if (k >= it.nkeys) return;
  float* at = weight_at(w, it, it.key0 + k);
  if (at != nullptr) *at += sum;
}

struct WeighLayout {
  size_t item, next, total;
};
WeighLayout weigh_layout() {
  WeighLayout L{};
  L.item = 256;  // the status word
  L.next = L.item + ((kMaxWeighCtas * sizeof(WeighItem) + 255) & ~(size_t)255);
  L.total = L.next + (size_t)kMaxWeighCtas * kWeighSpan * sizeof(float);
  return L;
}

bool sizes_ok(int32_t tokens, int32_t batch, int32_t h_q, int32_t h_kv) {
  return tokens >= 0 && batch >= 1 && h_q >= 1 && h_kv >= 1 && h_q % h_kv == 0 && h_q <= (1 << 16);
}

}  // namespace
}  // namespace ecokv

using namespace ecokv;

extern "C" {

size_t ecokv_weigh_workspace_size(int32_t tokens, int32_t batch, int32_t h_q, int32_t h_kv, ecokv_dtype dtype) {
  if (!sizes_ok(tokens, batch, h_q, h_kv) || (dtype != ECOKV_F32 && dtype != ECOKV_BF16)) return 0;
  return weigh_layout().total;
}

ecokv_status ecokv_weigh(const ecokv_weigh_params* p, ecokv_dtype dtype, const void* q, const float* lse,
                         const ecokv_prefix* prefix, const ecokv_pages* cache, const int32_t* starts,
                         const ecokv_weights* prefix_weights, const ecokv_weights* weights, void* ws, size_t ws_bytes,
                         void* stream) {
  if (p == nullptr || !sizes_ok(p->tokens, p->batch, p->h_q, p->h_kv) || p->d < 1) return ECOKV_ERR_INVALID_ARG;
  if (dtype != ECOKV_F32 && dtype != ECOKV_BF16) return ECOKV_ERR_INVALID_ARG;
  const size_t e = dtype == ECOKV_F32 ? 4 : 2;
  if ((p->flags & ~(ECOKV_FLAG_FORCE_SIMT | ECOKV_FLAG_TEST_STALL)) != 0u || !isfinite(p->scale) ||
      !isfinite(p->decay) || p->decay < 0.f)
    return ECOKV_ERR_INVALID_ARG;
  const bool tc = dtype == ECOKV_BF16 && (p->flags & ECOKV_FLAG_FORCE_SIMT) == 0u;
  if ((p->flags & ECOKV_FLAG_TEST_STALL) != 0u && !tc) return ECOKV_ERR_UNSUPPORTED;  // the waits are on that path
  if (p->d != kD || p->h_q / p->h_kv > kMaxGroup) return ECOKV_ERR_UNSUPPORTED;
  if (p->tokens == 0) return ECOKV_OK;
  if (!q || !lse || !aligned16(q) || ((uintptr_t)lse & 3u)) return ECOKV_ERR_INVALID_ARG;
  if (p->q_token <= 0 || p->q_head <= 0 || !stride_ok(p->q_token, e) || !stride_ok(p->q_head, e))
    return ECOKV_ERR_INVALID_ARG;
  WeighArgs w{};
  AttendArgs& a = w.a;
  if (prefix != nullptr && prefix->rows != 0) {
    if (prefix->rows < 0 || !prefix->k || !aligned16(prefix->k) || ((uintptr_t)prefix->head_off & 3u) ||
        prefix->row_stride <= 0 || !stride_ok(prefix->row_stride, e) ||
        (!prefix->head_off && (prefix->head_stride <= 0 || !stride_ok(prefix->head_stride, e))))
      return ECOKV_ERR_INVALID_ARG;
    if (prefix->rows > kMaxN) return ECOKV_ERR_UNSUPPORTED;
    if (prefix_weights == nullptr || !prefix_weights->w || ((uintptr_t)prefix_weights->w & 3u) ||
        prefix_weights->slot_stride <= 0 || (!prefix->head_off && prefix_weights->head_stride <= 0))
      return ECOKV_ERR_INVALID_ARG;
    a.prefix = *prefix;
    w.pw = *prefix_weights;
  }
  if (cache != nullptr) {
    ecokv_pages c = *cache;
    c.v = c.k;  // (not read)
    const ecokv_status st = check_pages(&c, p->batch, dtype);
    if (st != ECOKV_OK) return st;
    if ((uintptr_t)starts & 3u || (starts == nullptr && p->tokens != p->batch)) return ECOKV_ERR_INVALID_ARG;
    if (weights == nullptr || !weights->w || ((uintptr_t)weights->w & 3u) || weights->page_stride <= 0 ||
        weights->head_stride <= 0 || weights->slot_stride <= 0)
      return ECOKV_ERR_INVALID_ARG;
    a.cache = c;
    a.has_cache = 1;
    a.page_shift = __builtin_ctz((unsigned)cache->page_size);
    a.cap = cache->page_size * cache->table_stride;
    a.starts = starts;
    w.w = *weights;
  }
  a.q = q;
  a.q_token = p->q_token;
  a.q_head = p->q_head;
  a.tokens = p->tokens;
  a.batch = p->batch;
  a.h_q = p->h_q;
  a.h_kv = p->h_kv;
  a.g = p->h_q / p->h_kv;
  a.stall = (p->flags & ECOKV_FLAG_TEST_STALL) ? 1 : 0;
  const double scale = p->scale > 0.f ? (double)p->scale : 1.0 / sqrt((double)kD);
  a.scale_log2 = (float)(1.4426950408889634 * scale);
  a.timeout_ns = (p->timeout_us ? (unsigned long long)p->timeout_us : 2000000ull) * 1000ull;
  w.lse = lse;
  w.decay = p->decay;
  w.span = tc ? kWeighSpan : 128;
  w.span_log2 = tc ? 8 : 7;
  static_assert(kWeighSpan == 1 << 8, "span_log2");
  w.tpt[0] = (tc ? 128 : 64) / a.g;
  // a sequence's own row tiles have room for twice the mean of its tokens: what is copied and
  // multiplied of a decode step's single rows is no more than they are
  const int mean = a.starts != nullptr ? (a.tokens - 1) / a.batch + 1 : 1;
  auto tiles = [](int ntok, int tpt) { return (ntok - 1) / tpt + 1; };  // (ntok + tpt may not be an int)
  if (!tc && a.tokens > w.tpt[0]) w.tpt[0] = tiles(a.tokens, tiles(a.tokens, w.tpt[0]));  // equal ones
  w.tpt[1] = a.starts != nullptr && mean < (w.tpt[0] + 1) / 2 ? 2 * mean : a.starts != nullptr ? w.tpt[0] : 1;
  // (a unit: about 600 cycles of a CTA, an item of 256 keys with one row tile 5 of them, each row
  // tile of 128 rows 4; on CUDA cores: about 1700, 128 keys two of them and a tile of 64 rows 22)
  for (int k = 0; k < 2; ++k) w.unit[k] = div_up((a.tokens < w.tpt[k] ? a.tokens : w.tpt[k]) * a.g, tc ? 32 : 3);
  w.lead = tc ? 4 : 2;
  w.whole = 24;
  // (the units of the largest items that there can be)
  auto units = [&](int source, int ntok) { return w.lead + (double)w.unit[source] * tiles(ntok, w.tpt[source]); };
  const bool cut = (a.prefix.rows > 0 && units(0, a.tokens) > w.whole) ||
                   (a.has_cache && units(1, a.starts != nullptr ? a.tokens : 1) > w.whole);
  // (a cut item's tile at least: no CTA between its first and last is without a tile of it)
  w.least = cut ? (w.unit[0] > w.unit[1] ? w.unit[0] : w.unit[1]) : 1;
  // Units of all items, counted in 31 bits by the kernels: as many as there can be of the sequences'
  // slots.  (A sequence's tokens make a row tile more than their share.)
  const double items = div_up(a.cap, w.span), of_prefix = div_up(a.prefix.rows, w.span);
  const double row_tiles = tiles(a.tokens, w.tpt[1]) + (double)a.batch;
  const double own = items * (a.batch * (double)w.lead + row_tiles * w.unit[1]);
  if (a.h_kv * (of_prefix * units(0, a.tokens) + own) > 0x7fffffff) return ECOKV_ERR_UNSUPPORTED;
  const WeighLayout L = weigh_layout();
  if (ws == nullptr || !aligned16(ws) || ws_bytes < L.total) return ECOKV_ERR_WORKSPACE;
  a.P = attend_sms() * (tc ? 1 : 2);
  char* base = static_cast<char*>(ws);
  a.status = reinterpret_cast<unsigned*>(base);
  w.next_item = reinterpret_cast<WeighItem*>(base + L.item);
  w.next = reinterpret_cast<float*>(base + L.next);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.prefix.rows == 0 && !a.has_cache) return ECOKV_OK;
  if ((tc ? launch_weigh_tc(w, s) : launch_weigh_simt(w, dtype, s)) != cudaSuccess) return ECOKV_ERR_CUDA;
  if (!cut) return ECOKV_OK;
  return launch_behind(weigh_join_kernel, (unsigned)a.P, kWeighSpan, 0, s, w) == cudaSuccess ? ECOKV_OK : ECOKV_ERR_CUDA;
}

}  // extern "C"
