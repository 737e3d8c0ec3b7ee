// The walks over a call's items (csrc/attend.cuh, csrc/weigh.cuh) on the CPU: the 32 lanes of
// a warp are contexts that take turns, each running up to its next warp-wide operation.
//
//   walk_host weigh|attend < numbers     (see main)
//
// prints an item a line, CTA by CTA.  The object that a walk fills is a fresh one for each
// item, all its bytes 0x7b before: what next() returns may not rest on it.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <ucontext.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#undef __launch_bounds__
#define __launch_bounds__(...)

namespace warp {
constexpr size_t kStack = 256 * 1024;
ucontext_t back, at[32];
char stacks[32][kStack];
bool done[32];
int lane;
unsigned long long turn[32];  // warp-wide operations so far
unsigned long long slot[2][32];
void (*body)(int);

void start() {
  body(lane);
  done[lane] = true;
  swapcontext(&at[lane], &back);
}
// Every lane's value of this operation.
const unsigned long long* share(unsigned long long v) {
  const int me = lane;
  const unsigned long long k = turn[me]++ & 1;
  slot[k][me] = v;
  swapcontext(&at[me], &back);
  return slot[k];  // (the other half is written meanwhile)
}
void run(void (*f)(int)) {
  body = f;
  for (int i = 0; i < 32; ++i) {
    done[i] = false;
    turn[i] = 0;
    getcontext(&at[i]);
    at[i].uc_stack.ss_sp = stacks[i];
    at[i].uc_stack.ss_size = kStack;
    at[i].uc_link = &back;
    makecontext(&at[i], start, 0);
  }
  for (bool more = true; more;) {
    more = false;
    int ended = 0;
    for (lane = 0; lane < 32; ++lane) {
      if (!done[lane]) swapcontext(&back, &at[lane]);
      ended += done[lane];
    }
    more = ended < 32;
    if (more && ended > 0) {
      std::fprintf(stderr, "some lanes have left the others\n");
      std::exit(3);
    }
  }
}
}  // namespace warp

inline int __shfl_sync(unsigned, int v, int from) { return (int)warp::share((unsigned)v)[from & 31]; }
inline int __shfl_up_sync(unsigned, int v, int d) {
  const int me = warp::lane;
  const unsigned long long* all = warp::share((unsigned)v);
  return (int)all[me >= d ? me - d : me];
}
inline unsigned __ballot_sync(unsigned, bool p) {
  const unsigned long long* all = warp::share(p);
  unsigned m = 0;
  for (int i = 0; i < 32; ++i) m |= (unsigned)all[i] << i;
  return m;
}
inline unsigned __reduce_add_sync(unsigned, unsigned v) {
  const unsigned long long* all = warp::share(v);
  unsigned s = 0;
  for (int i = 0; i < 32; ++i) s += (unsigned)all[i];
  return s;
}
inline int __ffs(unsigned v) { return __builtin_ffs((int)v); }
inline unsigned atomicCAS(unsigned* p, unsigned expected, unsigned v) {
  const unsigned old = *p;
  if (old == expected) *p = v;
  return old;
}
using std::max;
using std::min;

#include "weigh.cuh"

namespace ecokv {

static WeighArgs w{};
static int cta;
static unsigned status[2];
static std::vector<int> plan, starts, lengths, head_off;

template <typename Item>
Item poisoned() {
  Item it;
  std::memset(&it, 0x7b, sizeof it);
  return it;
}

static void weigh_lane(int lane) {
  WeighWalk walk;
  walk.begin(w, cta, lane, cta == 0);
  while (true) {
    WeighItem it = poisoned<WeighItem>();
    if (!walk.next(w, it)) break;
    if (lane == 0)
      std::printf("%d %d %d %d %d %d %d %d %d %d %d %d\n", cta, it.source, it.head, it.seq, it.key0, it.nkeys, it.tok0,
                  it.ntok, it.base, it.row0, it.tile0, it.ntiles);
  }
}

static void attend_lane(int lane) {
  Walk walk;
  walk.begin(w.a, cta, lane);
  while (true) {
    Item it = poisoned<Item>();
    if (!walk.next(w.a, it)) break;
    if (lane == 0)
      std::printf("%d %d %d %d %d %d %d %d %d %d %d %d\n", cta, it.source, it.head, it.seq, it.tok0, it.ntok, it.lim0,
                  it.slope, it.vis, it.row0, it.tile0, it.ntiles);
  }
}

static int number() {
  int x = 0;
  if (std::scanf("%d", &x) != 1) std::exit(2);
  return x;
}
static void list(std::vector<int>& x, int n) {
  x.resize(n);
  for (int& v : x) v = number();
}

}  // namespace ecokv

// P first_cta last_cta h_kv tokens batch rows cap has_cache with_starts with_offsets, then
//   weigh: span_log2 tpt0 tpt1 unit0 unit1 lead whole least
//   attend: tpt span lead tree
// then lengths [batch], starts [batch + 1], offsets [h_kv + 1], each where the call has them.
int main(int argc, char** argv) {
  using namespace ecokv;
  if (argc != 2) return 2;
  const bool weighing = std::strcmp(argv[1], "weigh") == 0;
  AttendArgs& a = w.a;
  a.P = number();
  const int first = number(), last = number();
  a.h_kv = number();
  a.tokens = number();
  a.batch = number();
  a.prefix.rows = number();
  a.cap = number();
  a.has_cache = number();
  const int with_starts = number(), with_offsets = number();
  a.status = status;
  if (weighing) {
    w.span_log2 = number();
    w.span = 1 << w.span_log2;
    for (int& x : w.tpt) x = number();
    for (int& x : w.unit) x = number();
    w.lead = number();
    w.whole = number();
    w.least = number();
  } else {
    a.tpt = number();
    a.span = number();
    a.lead = number();
    static const uint32_t any = 0;
    if (number()) a.mask = &any;
    a.groups = (a.tokens - 1) / a.span + 1;
    a.last = a.tokens - (a.groups - 1) * a.span;
    plan.resize(PLAN_HEADS + a.h_kv + a.batch);
    a.plan = plan.data();
  }
  if (a.has_cache) {
    list(lengths, a.batch);
    a.cache.lengths = lengths.data();
  }
  if (with_starts) {
    list(starts, a.batch + 1);
    a.starts = starts.data();
  }
  if (with_offsets) {
    list(head_off, a.h_kv + 1);
    a.prefix.head_off = head_off.data();
  }
  for (cta = first; cta <= last; ++cta) warp::run(weighing ? weigh_lane : attend_lane);
  std::printf("status %u\n", status[0]);
  return 0;
}
