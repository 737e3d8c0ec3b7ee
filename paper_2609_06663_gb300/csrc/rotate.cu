// ecokv_rotate and ecokv_append: per-head RMS norm and rotary positions of query
// and key rows, into rows of any strides or into the slots of a paged cache.
//
// A row is 128 elements, held by eight lanes of sixteen.  Lane c holds the pairs
// of frequencies 8c .. 8c + 7 in either layout: elements 8c.. and rot/2 + 8c.. (half)
// or 16c .. 16c + 15 (interleaved), so that a rotation stays within a lane, its loads
// are 16 bytes wide, and the norm's sum is three shuffles away.  A warp takes a run
// of rows in the order of tokens and heads, four at a time: its reads are whole
// kilobytes side by side where heads are.  (With a run for each eight lanes 32768
// tokens of 28 + 4 heads took 97 us.)  All runs are equally long and resident at
// once.  The warp forms the sines and cosines of each token that it meets once,
// two a lane, and hands them round.
//
// The angle.  position * inv_freq / 2 pi mod 1 is position * turns mod 2^64 with
// turns = inv_freq / 2 pi in units of 2^-64: the product wraps as the angle does, so
// the only error is the frequency's own (2^-53 relative) and the last rounding to
// 24 bits.  In fp32 position * inv_freq alone would be off by 2^-24 of the
// position, 0.008 rad at 131072.
//
// Bound by HBM: every row is read and written once.  32768 tokens of 28 + 4 heads, the
// keys to a layout of their own: 92 us, 5.8 TB/s, 86 % of the measured copy.  fp32 rows
// and interleaved bf16 ones are at 64 %: a lane then has 32 or 64 bytes side by side, of
// which a copy or a store takes 16, so that every sector comes twice, half of it used
// each time (16.8 million sectors read from L2 for 8.4 million of data; the same prompt
// interleaved 124 us, 32768 tokens of 8 + 8 fp32 heads 124).

#include <math.h>
#include <string.h>

#include "attend.cuh"
#include "decode_ptx.cuh"

namespace ecokv {
namespace {

constexpr int kGroup = 8;                // lanes a row
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
// 32768 tokens of 28 + 4 bf16 heads / 48 questions into pages / 5003 tokens of 8 + 8
// fp32 heads, us: 2 CTAs an SM and 2 steps 92.5 / 45.6 / 21.6, 3 steps 95.7 / 50.1 /
// 22.5; 3 CTAs 98.0 / 50.3 / 21.5; 4 CTAs 99.4 / 53.2 / 23.3 (more in flight only has
// reads and writes meet in DRAM more often).
constexpr int kResident = 2;             // CTAs an SM
constexpr int kDepth = 2;                // steps of 2 KB whose copies a warp has in flight or at hand

struct RowSet {
  const void* x;
  void* y;
  int64_t x_token, x_head, y_token, y_head;
  const void* norm;
  int heads;
};

struct RotateArgs {
  ecokv_rotary r;          // rot_dim 0: no rotation
  RowSet q, k, v;          // v: append only, copied
  const int32_t* positions;
  int tokens;
  int run;                 // rows (of q, k and v together) a warp takes
  float eps;
  // append
  ecokv_pages cache;
  const int32_t* starts;
  int batch;
  int page_shift;
  unsigned* status;
};

template <typename T>
struct Vec;  // 8 elements, in 16-byte pieces
template <>
struct Vec<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = v; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Vec<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = a;
    reinterpret_cast<float4*>(p)[1] = b;
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    a = make_float4(f[0], f[1], f[2], f[3]);
    b = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// Norm and rotation of one row; every lane of its group takes part.
template <typename T, bool kInter>
__device__ __forceinline__ void turn_row(Vec<T>& v0, Vec<T>& v1, const float (&cs)[8], const float (&sn)[8],
                                         bool turned, bool norm, const Vec<T>& w0, const Vec<T>& w1, float eps) {
  float a[8], b[8];
  v0.get(a);
  v1.get(b);
  if (norm) {
    float ss = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      ss = fmaf(a[i], a[i], ss);
      s1 = fmaf(b[i], b[i], s1);
    }
    ss += s1;
#pragma unroll
    for (int o = 1; o < kGroup; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float inv = rsqrtf(ss * (1.f / kD) + eps);
    float wa[8], wb[8];
    w0.get(wa);
    w1.get(wb);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      a[i] = a[i] * inv * wa[i];
      b[i] = b[i] * inv * wb[i];
    }
  }
  if (turned) {
    if constexpr (kInter) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = a[2 * i], y = a[2 * i + 1], z = b[2 * i], t = b[2 * i + 1];
        a[2 * i] = x * cs[i] - y * sn[i];
        a[2 * i + 1] = y * cs[i] + x * sn[i];
        b[2 * i] = z * cs[4 + i] - t * sn[4 + i];
        b[2 * i + 1] = t * cs[4 + i] + z * sn[4 + i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = a[i], y = b[i];
        a[i] = x * cs[i] - y * sn[i];
        b[i] = y * cs[i] + x * sn[i];
      }
    }
  }
  v0.set(a);
  v1.set(b);
}

// The sequence of a warp's token, and the token's slot.
struct Slot {
  int b, start, n, len;  // sequence; its first token, tokens and slots
  int64_t page;
  int row;               // -1: none
};
__device__ __forceinline__ void load_sequence(const RotateArgs& a, Slot& s, int b) {
  s.b = b;
  s.start = b;
  s.n = 1;
  if (a.starts != nullptr) {
    s.start = a.starts[b];
    s.n = a.starts[b + 1] - s.start;
  }
  s.len = a.cache.lengths[b];
}
// ... of the warp's first token t: as many of starts[1 .. batch] as are <= t come before it.
__device__ __forceinline__ void first_sequence(const RotateArgs& a, Slot& s, int t, int lane) {
  int b = t;
  if (a.starts != nullptr) {
    b = 0;
    for (int j = lane; j < a.batch; j += 32) b += a.starts[1 + j] <= t ? 1 : 0;
    b = min((int)__reduce_add_sync(0xffffffffu, (unsigned)b), a.batch - 1);
  }
  load_sequence(a, s, b);
}
__device__ __forceinline__ void find_slot(const RotateArgs& a, Slot& s, int t) {
  const int i = t - s.start;
  const long long slot = (long long)s.len - s.n + i, col = slot >> a.page_shift;
  s.row = -1;
  s.page = 0;
  if (slot >= 0 && col < a.cache.table_stride && i >= 0 && i < s.n) {
    s.page = a.cache.table[(int64_t)s.b * a.cache.table_stride + col];
    if (s.page >= 0 && s.page < a.cache.n_pages) s.row = (int)(slot & (a.cache.page_size - 1));
  }
  if (s.row < 0 && a.status != nullptr) {
    if (atomicCAS(a.status, 0u, (unsigned)ECOKV_ERR_DEVICE_INDEX) == 0u) a.status[1] = (unsigned)s.b;
  }
}

__device__ __forceinline__ void copy16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(dst)), "l"(src) : "memory");
}

// A warp's run of rows in steps: rows r .. r + n - 1 of token t, of one tensor.
template <int kRows>
struct Steps {
  int t, r, left;
  __device__ __forceinline__ int rows(int q_end, int k_end, int v_end) const {
    return min(min(kRows, left), (r < q_end ? q_end : r < k_end ? k_end : v_end) - r);
  }
  // whether a new token begins
  __device__ __forceinline__ bool next(int n, int v_end) {
    left -= n;
    r += n;
    if (r < v_end) return false;
    r = 0;
    ++t;
    return true;
  }
};

template <typename T, bool kInter, bool kAppend>
__global__ void __launch_bounds__(kThreads, kResident) rotate_kernel(const __grid_constant__ RotateArgs a) {
  constexpr int kPer = sizeof(T) == 2 ? 2 : 1;  // rows a lane has of a step
  constexpr int kVecs = 2 * kPer * (int)sizeof(Vec<T>) / 16;
  __shared__ uint4 ring[kWarps][kDepth][kVecs][32];
  // (the next kernel's launch may go ahead; this one's has, until here)
  ptx::grid_trigger();
  ptx::grid_wait();
  const int lane = threadIdx.x & 31, c = lane & (kGroup - 1), g = lane / kGroup;
  const int q_end = a.q.heads, k_end = q_end + a.k.heads, v_end = k_end + (kAppend ? a.v.heads : 0);
  const long long total = (long long)a.tokens * v_end;
  const long long first = ((long long)blockIdx.x * kWarps + threadIdx.x / 32) * a.run;
  if (first >= total) return;
  Steps<4 * kPer> take, done;
  done.left = (int)min((long long)a.run, total - first);
  done.t = (int)(first / v_end);
  done.r = (int)(first - (long long)done.t * v_end);
  take = done;
  const int F8 = a.r.rot_dim >> 4;  // lanes whose elements turn
  const bool turned = c < F8;
  // this lane's two eights of elements
  const int e0 = !kInter && turned ? 8 * c : 16 * c;
  const int e1 = !kInter && turned ? 8 * c + 8 * F8 : 16 * c + 8;
  uint4(*mine)[kVecs][32] = ring[threadIdx.x / 32];
  // this lane's pieces of the next step to memory of its own, kDepth - 1 steps ahead
  auto fetch = [&](int stage) {
    if (take.left > 0) {
      const int n = take.rows(q_end, k_end, v_end);
      const RowSet& s = take.r < q_end ? a.q : take.r < k_end ? a.k : a.v;
      const int h = take.r - (take.r < q_end ? 0 : take.r < k_end ? q_end : k_end) + g;
      const T* x = static_cast<const T*>(s.x) + (int64_t)take.t * s.x_token + (int64_t)h * s.x_head;
#pragma unroll
      for (int k = 0; k < kPer; ++k, x += 4 * s.x_head)
        if (g + 4 * k < n) {
          constexpr int kHalf = kVecs / kPer / 2;  // 16-byte pieces of an eight
#pragma unroll
          for (int i = 0; i < kHalf; ++i) {
            copy16(&mine[stage][2 * kHalf * k + i][lane], x + e0 + i * (8 / kHalf));
            copy16(&mine[stage][2 * kHalf * k + kHalf + i][lane], x + e1 + i * (8 / kHalf));
          }
        }
      take.next(n, v_end);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kDepth - 1; ++i) fetch(i);
  Slot at{};
  at.row = -1;
  if constexpr (kAppend) {
    first_sequence(a, at, done.t, lane);
    find_slot(a, at, done.t);
  }
  const int f0 = turned ? 8 * c + 2 * g : 0;  // the two frequencies of which this lane forms the sines
  const int* pos0 = a.positions + (F8 > 0 ? (int64_t)a.r.axis[f0] * a.tokens : 0);
  const int* pos1 = a.positions + (F8 > 0 ? (int64_t)a.r.axis[f0 + 1] * a.tokens : 0);
  const uint64_t turns[2] = {a.r.turns[f0], a.r.turns[f0 + 1]};
  int next_pos[2] = {0, 0};
  if (F8 > 0) {
    next_pos[0] = pos0[done.t];
    next_pos[1] = pos1[done.t];
  }
  float cs[8], sn[8];
  int64_t page = 0;
  int row = -1;
  bool fresh = true;
#pragma unroll 1
  for (int stage = 0; done.left > 0; stage = stage + 1 == kDepth ? 0 : stage + 1) {
    fetch(stage == 0 ? kDepth - 1 : stage - 1);
    if (fresh) {
      // a new token: its angles and slot, and loads for those of the one after it
      if (F8 > 0) {
        float s2[2], c2[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          // the upper 32 bits as a signed fraction of a turn: -1/2 .. 1/2, in half turns
          const uint64_t p = (uint64_t)(int64_t)next_pos[i];
          const int32_t ph = (int32_t)((p * turns[i] + 0x80000000ull) >> 32);
          sincospif((float)ph * 4.656612873077393e-10f, &s2[i], &c2[i]);
          s2[i] *= a.r.magnitude;
          c2[i] *= a.r.magnitude;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          cs[i] = __shfl_sync(0xffffffffu, c2[i & 1], (i >> 1) * kGroup + c);
          sn[i] = __shfl_sync(0xffffffffu, s2[i & 1], (i >> 1) * kGroup + c);
        }
      }
      const bool more = done.left > v_end - done.r;  // the run goes on to the next token
      const int tn = done.t + 1;
      if (F8 > 0 && more) {
        next_pos[0] = pos0[tn];
        next_pos[1] = pos1[tn];
      }
      if constexpr (kAppend) {
        page = at.page;
        row = at.row;
        if (more) {
          while (tn >= at.start + at.n && at.b + 1 < a.batch) load_sequence(a, at, at.b + 1);
          find_slot(a, at, tn);
        }
      }
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
    const int n = done.rows(q_end, k_end, v_end);
    const bool is_q = done.r < q_end, is_v = kAppend && done.r >= k_end;
    const RowSet& s = is_q ? a.q : a.k;
    const int h = done.r - (is_q ? 0 : is_v ? k_end : q_end) + g;
    const bool norm = !is_v && s.norm != nullptr;
    Vec<T> w0{}, w1{};
    if (norm) {
      w0.load(static_cast<const T*>(s.norm) + e0);
      w1.load(static_cast<const T*>(s.norm) + e1);
    }
    T* y = static_cast<T*>(s.y) + (int64_t)done.t * s.y_token;
    int64_t y_head = s.y_head;
    bool store = true;
    if (kAppend && !is_q) {
      y = static_cast<T*>(is_v ? a.cache.v : a.cache.k) + page * a.cache.page_stride +
          (int64_t)row * a.cache.slot_stride;
      y_head = a.cache.head_stride;
      store = row >= 0;
    }
    y += h * y_head;
#pragma unroll
    for (int k = 0; k < kPer; ++k, y += 4 * y_head) {
      Vec<T> v[2];
#pragma unroll
      for (int i = 0; i < kVecs / kPer; ++i)
        reinterpret_cast<uint4*>(v)[i] = mine[stage][kVecs / kPer * k + i][lane];
      if (!is_v) turn_row<T, kInter>(v[0], v[1], cs, sn, turned, norm, w0, w1, a.eps);
      if (store && g + 4 * k < n) {
        v[0].store(y + e0);
        v[1].store(y + e1);
      }
    }
    fresh = done.next(n, v_end);
  }
}

bool rotary_ok(const ecokv_rotary& r) {
  if (r.rot_dim < 16 || r.rot_dim > kD || r.rot_dim % 16 != 0) return false;
  if (r.layout != ECOKV_ROTARY_HALF && r.layout != ECOKV_ROTARY_INTERLEAVED) return false;
  if (r.axes < 1 || r.axes > ECOKV_ROTARY_AXES || !isfinite(r.magnitude)) return false;
  for (int f = 0; f < r.rot_dim / 2; ++f)
    if (r.axis[f] >= r.axes) return false;
  return true;
}

// A row set with heads is complete and aligned; out: whether y is used.
bool rows_ok(const ecokv_rows* s, size_t e, bool out) {
  if (s == nullptr) return true;
  if (s->heads < 1 || s->heads > (1 << 16) || !s->x || !aligned16(s->x) || !aligned16(s->norm)) return false;
  if (!stride_ok(s->x_token, e) || !stride_ok(s->x_head, e)) return false;
  if (out && (!s->y || !aligned16(s->y) || s->y_token <= 0 || s->y_head <= 0 || !stride_ok(s->y_token, e) ||
              !stride_ok(s->y_head, e)))
    return false;
  return true;
}

RowSet row_set(const ecokv_rows* s) {
  RowSet r{};
  if (s == nullptr) return r;
  r.x = s->x;
  r.y = s->y;
  r.x_token = s->x_token;
  r.x_head = s->x_head;
  r.y_token = s->y_token;
  r.y_head = s->y_head;
  r.norm = s->norm;
  r.heads = s->heads;
  return r;
}

template <typename T, bool kAppend>
cudaError_t launch(const RotateArgs& a, cudaStream_t st) {
  const long long rows = (long long)a.tokens * (a.q.heads + a.k.heads + a.v.heads);
  const long long warps = (rows + a.run - 1) / a.run;
  const unsigned grid = (unsigned)((warps + kWarps - 1) / kWarps);
  if (a.r.rot_dim > 0 && a.r.layout == ECOKV_ROTARY_INTERLEAVED)
    return launch_behind(rotate_kernel<T, true, kAppend>, grid, kThreads, 0, st, a);
  return launch_behind(rotate_kernel<T, false, kAppend>, grid, kThreads, 0, st, a);
}

// Rows a warp takes: as many as leave every warp resident (152 SMs), so that the last
// of them ends with the others, and four at least.
void set_run(RotateArgs& a, int heads) {
  const long long rows = (long long)a.tokens * heads, warps = 152ll * kResident * kWarps;
  const long long run = (rows + warps - 1) / warps;
  a.run = (int)(run > 4 ? run : 4);
}

ecokv_status common(RotateArgs& a, const ecokv_rotary* r, const int32_t* positions, int32_t tokens, float eps) {
  if (tokens < 0 || !(eps >= 0.f) || !isfinite(eps)) return ECOKV_ERR_INVALID_ARG;
  if (r != nullptr) {
    if (!rotary_ok(*r) || positions == nullptr || ((uintptr_t)positions & 3u)) return ECOKV_ERR_INVALID_ARG;
    a.r = *r;
  }
  a.positions = positions;
  a.tokens = tokens;
  a.eps = eps;
  return ECOKV_OK;
}

bool too_many(int32_t tokens, long long heads) { return (long long)tokens * heads > 1ll << 31; }

}  // namespace
}  // namespace ecokv

using namespace ecokv;

extern "C" {

ecokv_status ecokv_rotary_set(ecokv_rotary* r, int32_t rot_dim, int32_t layout, const double* inv_freq,
                              float magnitude) {
  if (r == nullptr || inv_freq == nullptr) return ECOKV_ERR_INVALID_ARG;
  ecokv_rotary n;
  memset(&n, 0, sizeof(n));
  n.rot_dim = rot_dim;
  n.layout = layout;
  n.axes = 1;
  n.magnitude = magnitude;
  if (!rotary_ok(n)) return ECOKV_ERR_INVALID_ARG;
  for (int f = 0; f < rot_dim / 2; ++f) {
    if (!isfinite(inv_freq[f])) return ECOKV_ERR_INVALID_ARG;
    const double turns = inv_freq[f] / 6.283185307179586476925;
    const double x = (turns - floor(turns)) * 18446744073709551616.0;  // exact: a power of two
    n.turns[f] = x >= 18446744073709551616.0 ? 0 : (uint64_t)x;
  }
  *r = n;
  return ECOKV_OK;
}

ecokv_status ecokv_rotary_init(ecokv_rotary* r, int32_t rot_dim, int32_t layout, double base, int32_t scaling,
                               double factor, int32_t original) {
  if (r == nullptr || rot_dim < 16 || rot_dim > kD || rot_dim % 16 != 0) return ECOKV_ERR_INVALID_ARG;
  if (!(base > 0.0) || base == 1.0 || !isfinite(base)) return ECOKV_ERR_INVALID_ARG;
  if (scaling < ECOKV_ROTARY_NONE || scaling > ECOKV_ROTARY_YARN) return ECOKV_ERR_INVALID_ARG;
  if (scaling != ECOKV_ROTARY_NONE && (!(factor > 0.0) || !isfinite(factor))) return ECOKV_ERR_INVALID_ARG;
  if (scaling == ECOKV_ROTARY_YARN && original < 1) return ECOKV_ERR_INVALID_ARG;
  double freq[kD / 2];
  if (scaling == ECOKV_ROTARY_NTK) base *= pow(factor, rot_dim / (rot_dim - 2.0));
  for (int f = 0; f < rot_dim / 2; ++f) freq[f] = pow(base, -2.0 * f / rot_dim);
  float magnitude = 1.f;
  if (scaling == ECOKV_ROTARY_LINEAR)
    for (int f = 0; f < rot_dim / 2; ++f) freq[f] /= factor;
  if (scaling == ECOKV_ROTARY_YARN) {
    // pair whose wavelength is original / turns: original inv_freq = 2 pi turns
    const double pi2 = 6.283185307179586476925, lb = 2.0 * log(base);
    double lo = floor(rot_dim * log(original / (pi2 * 32.0)) / lb);
    double hi = ceil(rot_dim * log(original / pi2) / lb);
    lo = lo > 0.0 ? lo : 0.0;
    hi = hi < rot_dim - 1.0 ? hi : rot_dim - 1.0;
    const double width = hi - lo > 1e-3 ? hi - lo : 1e-3;
    for (int f = 0; f < rot_dim / 2; ++f) {
      double w = (f - lo) / width;
      w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
      freq[f] = freq[f] / factor * w + freq[f] * (1.0 - w);
    }
    magnitude = (float)(0.1 * log(factor) + 1.0);
  }
  return ecokv_rotary_set(r, rot_dim, layout, freq, magnitude);
}

ecokv_status ecokv_rotary_sections(ecokv_rotary* r, const int32_t* counts, int32_t axes) {
  if (r == nullptr || counts == nullptr || axes < 1 || axes > ECOKV_ROTARY_AXES) return ECOKV_ERR_INVALID_ARG;
  if (r->rot_dim < 16 || r->rot_dim > kD || r->rot_dim % 16 != 0) return ECOKV_ERR_INVALID_ARG;
  long long sum = 0;
  for (int x = 0; x < axes; ++x) {
    if (counts[x] < 0) return ECOKV_ERR_INVALID_ARG;
    sum += counts[x];
  }
  if (sum != r->rot_dim / 2) return ECOKV_ERR_INVALID_ARG;
  int f = 0;
  for (int x = 0; x < axes; ++x)
    for (int i = 0; i < counts[x]; ++i) r->axis[f++] = (uint8_t)x;
  r->axes = axes;
  return ECOKV_OK;
}

ecokv_status ecokv_rotate(const ecokv_rotary* r, ecokv_dtype dtype, const ecokv_rows* q, const ecokv_rows* k,
                          const int32_t* positions, int32_t tokens, float eps, void* stream) {
  if (dtype != ECOKV_F32 && dtype != ECOKV_BF16) return ECOKV_ERR_INVALID_ARG;
  if (tokens == 0) return ECOKV_OK;  // (tensors of no rows may have no address)
  const size_t e = dtype == ECOKV_F32 ? 4 : 2;
  if (!rows_ok(q, e, true) || !rows_ok(k, e, true)) return ECOKV_ERR_INVALID_ARG;
  RotateArgs a{};
  const ecokv_status st = common(a, r, positions, tokens, eps);
  if (st != ECOKV_OK) return st;
  a.q = row_set(q);
  a.k = row_set(k);
  const int heads = a.q.heads + a.k.heads;
  if (too_many(tokens, heads)) return ECOKV_ERR_UNSUPPORTED;
  if (heads == 0) return ECOKV_OK;
  set_run(a, heads);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t err = dtype == ECOKV_F32 ? launch<float, false>(a, s) : launch<__nv_bfloat16, false>(a, s);
  return err == cudaSuccess ? ECOKV_OK : ECOKV_ERR_CUDA;
}

ecokv_status ecokv_append(const ecokv_rotary* r, ecokv_dtype dtype, const ecokv_rows* q, const ecokv_rows* k,
                          const ecokv_rows* v, const ecokv_pages* cache, const int32_t* positions,
                          const int32_t* starts, int32_t tokens, int32_t batch, float eps, void* ws,
                          size_t ws_bytes, void* stream) {
  if (dtype != ECOKV_F32 && dtype != ECOKV_BF16) return ECOKV_ERR_INVALID_ARG;
  if (tokens == 0) return ECOKV_OK;
  const size_t e = dtype == ECOKV_F32 ? 4 : 2;
  if (k == nullptr || v == nullptr || !rows_ok(q, e, true) || !rows_ok(k, e, false) || !rows_ok(v, e, false))
    return ECOKV_ERR_INVALID_ARG;
  if (k->heads != v->heads || v->norm != nullptr) return ECOKV_ERR_INVALID_ARG;
  ecokv_status st = check_pages(cache, batch, dtype);
  if (st != ECOKV_OK) return st;
  if ((uintptr_t)starts & 3u || (starts == nullptr && tokens != batch)) return ECOKV_ERR_INVALID_ARG;
  if (ws != nullptr && (!aligned16(ws) || ws_bytes < 256)) return ECOKV_ERR_WORKSPACE;
  RotateArgs a{};
  st = common(a, r, positions, tokens, eps);
  if (st != ECOKV_OK) return st;
  a.q = row_set(q);
  a.k = row_set(k);
  a.v = row_set(v);
  const int heads = a.q.heads + a.k.heads + a.v.heads;
  if (too_many(tokens, heads)) return ECOKV_ERR_UNSUPPORTED;
  a.cache = *cache;
  a.starts = starts;
  a.batch = batch;
  a.page_shift = __builtin_ctz((unsigned)cache->page_size);
  a.status = static_cast<unsigned*>(ws);
  set_run(a, heads);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t err = dtype == ECOKV_F32 ? launch<float, true>(a, s) : launch<__nv_bfloat16, true>(a, s);
  return err == cudaSuccess ? ECOKV_OK : ECOKV_ERR_CUDA;
}

}  // extern "C"
