// Drafted tokens: the mask of a tree (ecokv_tree_mask), and the rows of the accepted ones
// (ecokv_commit).

#include "cache_move.cuh"

namespace ecokv {
namespace {

// Tokens of sequence b, clamped to the call's.
__device__ __forceinline__ int2 tokens_of(const int32_t* starts, int b, int tokens, unsigned* status) {
  const int s0 = starts ? starts[b] : b, s1 = starts ? starts[b + 1] : b + 1;
  const int from = min(max(s0, 0), tokens), n = min(max(s1, from), tokens) - from;
  if (from != s0 || from + n != s1) flag(status, (unsigned)b);
  return make_int2(from, n);
}

// Ancestors by doubling within each 64 tokens (a word of the mask): `seen` bits of the
// word and `up`, the ancestor that `seen` ends before, are joined with those of `up` six
// times; then a token's word of any lower 64 is `seen` of the first of its ancestors
// there, found hop by hop.  Latency bounds it: one CTA a sequence, the tree in shared
// memory (25 drafts 1.7 us on the device, 64 trees of up to 256 2.7).
constexpr int kMaxWords = 64;

__global__ void tree_mask_kernel(const int32_t* parents, const int32_t* starts, int tokens, uint64_t* mask, int words,
                                 unsigned* status) {
  extern __shared__ uint64_t seen[];  // [64 words], then up
  int* up = reinterpret_cast<int*>(seen + 64 * words);
  ptx::grid_trigger();
  ptx::grid_wait();
  const int b = blockIdx.x;
  const int2 t = tokens_of(starts, b, tokens, threadIdx.x == 0 ? status : nullptr);
  const int n = min(t.y, 64 * words);
  if (t.y > n && threadIdx.x == 0) flag(status, (unsigned)b);
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    int p = parents[t.x + i];
    if (p < -1 || p >= i) {
      flag(status, (unsigned)(t.x + i));
      p = -1;
    }
    up[i] = p;
    seen[i] = 1ull << (i & 63);
  }
  __syncthreads();
  for (int d = 1; d < 64 && d < n; d *= 2) {
    // (64 tokens are two of a warp's, or a thread's own: they are read before any is written)
    for (int i0 = 0; i0 < n; i0 += blockDim.x) {
      const int i = i0 + threadIdx.x;
      uint64_t s = 0;
      int u = -1;
      const bool more = i < n && (u = up[i]) >= (i & ~63);
      if (more) {
        s = seen[u];
        u = up[u];
      }
      __syncthreads();
      if (more) {
        seen[i] |= s;
        up[i] = u;
      }
      __syncthreads();
    }
  }
  for (int i = threadIdx.x; i < t.y; i += blockDim.x) {
    uint64_t* row = mask + (int64_t)(t.x + i) * words;
    int at = i < n ? i : -1;
    for (int w = words - 1; w >= 0; --w) {
      uint64_t x = 0;
      if (at >= 0 && at >> 6 == w) {
        x = seen[at];
        at = up[at];
      }
      row[w] = x;
    }
  }
}

// The rows of the accepted drafts: one CTA a sequence, head and K or V, whose list every CTA
// checks for itself.  Latency bounds it: list, pages, rows (16 paths, 4 heads 3.1 us on
// the device; 64 of up to 256 drafts, 8 fp32 heads and weights 6.1).
struct CommitArgs {
  MoveArgs m;
  const int32_t* accepted;
  const int32_t* counts;
  const int32_t* starts;
  int32_t* lengths_out;  // NULL: another kernel's
  int stride, tokens, cap;
};

struct Path {
  int base, n;  // slots before the drafts, accepted ones
};

// All of the CTA's threads.
__device__ __forceinline__ Path read_path(const CommitArgs& a, int b) {
  unsigned* status = threadIdx.x == 0 ? a.m.status : nullptr;
  const int T = tokens_of(a.starts, b, a.tokens, status).y;
  const int len = a.m.from.lengths[b], L = min(max(len, 0), a.cap);
  if (L != len) flag(status, (unsigned)b);
  Path p;
  p.base = L - T;
  p.n = a.counts[b];
  const int32_t* list = a.accepted + (int64_t)b * a.stride;
  bool ok = p.base >= 0 && p.n >= 0 && p.n <= T && p.n <= a.stride;
  if (ok)
    for (int i = threadIdx.x; i < p.n; i += blockDim.x) {
      const int x = list[i], before = i > 0 ? list[i - 1] : -1;
      ok = ok && x > before && x < T;
    }
  if (!__syncthreads_and(ok)) {
    flag(status, (unsigned)b);
    p.base = max(p.base, 0);
    p.n = 0;
  }
  return p;
}

constexpr int kThreads = 256;

template <int E>
__global__ void __launch_bounds__(kThreads, 4) commit_kernel(const __grid_constant__ CommitArgs a) {
  ptx::grid_trigger();
  ptx::grid_wait();
  const int unit = blockIdx.x;
  const int kv = unit & 1, h = (unit >> 1) % a.m.h_kv, b = (unit >> 1) / a.m.h_kv;
  const Path p = read_path(a, b);
  const int32_t* list = a.accepted + (int64_t)b * a.stride;
  move_rows<E, kThreads>(a.m, b, h, kv, 0, 0, p.n, p.base, [=](int i) { return p.base + list[i]; });
  if (a.lengths_out != nullptr && h == 0 && kv == 0 && threadIdx.x == 0) a.lengths_out[b] = p.base + p.n;
}

// The lengths alone, once nothing reads the old ones any more.
__global__ void __launch_bounds__(64) commit_lengths_kernel(const __grid_constant__ CommitArgs a) {
  ptx::grid_trigger();
  ptx::grid_wait();
  const Path p = read_path(a, blockIdx.x);
  if (threadIdx.x == 0) a.lengths_out[blockIdx.x] = p.base + p.n;
}

}  // namespace
}  // namespace ecokv

using namespace ecokv;

extern "C" {

ecokv_status ecokv_tree_mask(const int32_t* parents, const int32_t* starts, int32_t tokens, int32_t batch,
                             uint64_t* mask, int32_t words, void* ws, size_t ws_bytes, void* stream) {
  if (tokens < 0 || batch < 1 || words < 1) return ECOKV_ERR_INVALID_ARG;
  if (words > kMaxWords) return ECOKV_ERR_UNSUPPORTED;
  if (tokens == 0) return ECOKV_OK;
  if (!parents || !mask || ((uintptr_t)parents & 3u) || ((uintptr_t)mask & 7u) || ((uintptr_t)starts & 3u))
    return ECOKV_ERR_INVALID_ARG;
  if (starts == nullptr && tokens != batch) return ECOKV_ERR_INVALID_ARG;
  if (ws != nullptr && (!aligned16(ws) || ws_bytes < 256)) return ECOKV_ERR_WORKSPACE;
  const int room = 64 * words < tokens ? 64 * words : tokens;  // tokens a sequence may have in the mask
  const unsigned threads = room <= 32 ? 32 : room <= 64 ? 64 : room <= 128 ? 128 : room <= 256 ? 256 : 512;
  const size_t smem = (size_t)64 * words * (sizeof(uint64_t) + sizeof(int));
  static_assert(64 * kMaxWords * (sizeof(uint64_t) + sizeof(int)) <= 48 * 1024, "without an attribute");
  const cudaError_t e =
      launch_behind(tree_mask_kernel, (unsigned)batch, threads, smem, static_cast<cudaStream_t>(stream), parents,
                    starts, (int)tokens, mask, (int)words, static_cast<unsigned*>(ws));
  return e == cudaSuccess ? ECOKV_OK : ECOKV_ERR_CUDA;
}

ecokv_status ecokv_commit(ecokv_dtype dtype, const ecokv_pages* cache, int32_t h_kv, const int32_t* accepted,
                          int32_t stride, const int32_t* counts, const int32_t* starts, int32_t tokens, int32_t batch,
                          const ecokv_weights* weights, int32_t* lengths_out, void* ws, size_t ws_bytes,
                          void* stream) {
  if (dtype != ECOKV_F32 && dtype != ECOKV_BF16) return ECOKV_ERR_INVALID_ARG;
  if (tokens < 0 || h_kv < 1 || stride < 1) return ECOKV_ERR_INVALID_ARG;
  const ecokv_status st = check_pages(cache, batch, dtype);
  if (st != ECOKV_OK) return st;
  if (!accepted || !counts || ((uintptr_t)accepted & 3u) || ((uintptr_t)counts & 3u) || ((uintptr_t)starts & 3u) ||
      (starts == nullptr && tokens != batch) || !lengths_ok(cache->lengths, lengths_out, batch) ||
      !apart(counts, batch, lengths_out, batch) || !apart(accepted, (int64_t)batch * stride, lengths_out, batch) ||
      (starts != nullptr && !apart(starts, (int64_t)batch + 1, lengths_out, batch)))
    return ECOKV_ERR_INVALID_ARG;
  if (weights != nullptr && !weights_ok(weights)) return ECOKV_ERR_INVALID_ARG;
  if ((int64_t)batch * h_kv > 1 << 29) return ECOKV_ERR_UNSUPPORTED;
  if (ws != nullptr && (!aligned16(ws) || ws_bytes < 256)) return ECOKV_ERR_WORKSPACE;
  CommitArgs a{};
  a.m.from = a.m.to = *cache;
  if (weights != nullptr) a.m.w_from = a.m.w_to = *weights;
  a.m.from_shift = a.m.to_shift = __builtin_ctz((unsigned)cache->page_size);
  a.m.h_kv = h_kv;
  a.m.batch = batch;
  a.m.in_place = 1;
  a.m.status = static_cast<unsigned*>(ws);
  a.m.ctas = a.m.cluster = 1;
  a.accepted = accepted;
  a.counts = counts;
  a.starts = starts;
  a.stride = stride;
  a.tokens = tokens;
  a.cap = cache->page_size * cache->table_stride;
  const bool same = lengths_out == cache->lengths;
  a.lengths_out = same ? nullptr : lengths_out;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned grid = (unsigned)(2 * batch * h_kv);
  cudaError_t e = dtype == ECOKV_F32 ? launch_move(commit_kernel<4>, a.m, grid, kThreads, 0, s, a)
                                     : launch_move(commit_kernel<2>, a.m, grid, kThreads, 0, s, a);
  if (e == cudaSuccess && same) {
    a.lengths_out = lengths_out;
    e = launch_behind(commit_lengths_kernel, (unsigned)batch, 64, 0, s, a);
  }
  return e == cudaSuccess ? ECOKV_OK : ECOKV_ERR_CUDA;
}

}  // extern "C"
