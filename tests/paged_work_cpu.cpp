// The division of paged_attention's work (csrc/paged_work.h, csrc/cache_host.cpp) built for the CPU: the 64 lanes of one wave are 64 stacks that
// run in turn from one exchange between lanes to the next.
#include <setjmp.h>
#include <ucontext.h>

#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

struct Index {
  unsigned x;
};
static Index threadIdx, blockIdx, gridDim;
struct float2 {
  float x, y;
};
typedef uint16_t u16;
#define __device__
#define __forceinline__ inline

// ------------------------------------------------------------------------------------------------ one wave
struct Lane {
  ucontext_t start;
  jmp_buf at;
  bool begun, ended;
  std::vector<char> stack;
};
static Lane g_lanes[64];
static ucontext_t g_main;
static uint64_t g_said[2][64];
static int g_tag[2][64], g_turn[64];  // (tags: which exchange a lane is at)
static void (*g_body)();

static void apart() {
  fprintf(stderr, "the lanes went different ways\n");
  abort();
}
static void go_to(unsigned lane) {
  threadIdx.x = lane;
  Lane& l = g_lanes[lane];
  if (l.ended) apart();
  if (l.begun) _longjmp(l.at, 1);
  l.begun = true;
  setcontext(&l.start);
}
// Every lane says a value; returns what all have said.
__attribute__((noinline)) static const uint64_t* exchange(uint64_t x, int kind) {
  const unsigned lane = threadIdx.x;
  const int tag = g_turn[lane]++ << 3 | kind, turn = tag >> 3 & 1;
  g_said[turn][lane] = x;
  g_tag[turn][lane] = tag;
  if (!_setjmp(g_lanes[lane].at)) go_to((lane + 1) & 63);
  if (g_tag[turn][lane == 63 ? 0 : 63] != tag) apart();
  return g_said[turn];
}
static void lane_main() {
  g_body();
  g_lanes[threadIdx.x].ended = true;
  if (threadIdx.x == 63) setcontext(&g_main);
  go_to(threadIdx.x + 1);
}
static void run_wave(void (*body)()) {
  g_body = body;
  for (int i = 0; i < 64; ++i) {
    Lane& l = g_lanes[i];
    l.begun = l.ended = false;
    g_turn[i] = 0;
    if (l.stack.empty()) l.stack.resize(64 << 10);
    getcontext(&l.start);
    l.start.uc_stack.ss_sp = l.stack.data();
    l.start.uc_stack.ss_size = l.stack.size();
    l.start.uc_link = nullptr;
    makecontext(&l.start, lane_main, 0);
  }
  volatile bool done = false;
  getcontext(&g_main);
  if (done) return;
  done = true;
  go_to(0);
}

static int __builtin_amdgcn_readlane(int x, int lane) { return (int)exchange((uint32_t)x, 1)[lane & 63]; }
static int __builtin_amdgcn_readfirstlane(int x) { return (int)exchange((uint32_t)x, 2)[0]; }
static int __builtin_amdgcn_update_dpp(int old, int x, int ctrl, int rows, int banks, bool) {
  const uint64_t* said = exchange((uint32_t)x, 3);
  const int lane = threadIdx.x, row = lane >> 4;
  if (banks != 0xf) abort();
  if (!(rows >> row & 1)) return old;
  if (ctrl > 0x110 && ctrl < 0x120) return (lane & 15) >= (ctrl & 15) ? (int)said[lane - (ctrl & 15)] : old;  // from lanes below in a row
  if (ctrl == 0x142) return row ? (int)said[row * 16 - 1] : old;                                             // the last of the row below
  if (ctrl == 0x143) return row > 1 ? (int)said[31] : old;
  abort();
}
static uint64_t __ballot(bool x) {
  const uint64_t* said = exchange(x, 4);
  uint64_t all = 0;
  for (int i = 0; i < 64; ++i) all |= said[i] << i;
  return all;
}
static bool __any(bool x) { return __ballot(x) != 0; }
static int __popcll(uint64_t x) { return __builtin_popcountll(x); }
static int __ffsll(uint64_t x) { return __builtin_ffsll((long long)x); }
static unsigned __umulhi(unsigned a, unsigned b) { return (unsigned)(((uint64_t)a * b) >> 32); }
static int __float_as_int(float x) {
  int i;
  memcpy(&i, &x, 4);
  return i;
}
static float __int_as_float(int i) {
  float x;
  memcpy(&x, &i, 4);
  return x;
}
static float __uint_as_float(unsigned i) { return __int_as_float((int)i); }

#define NIMBLE_DEVICE_COMMON_H_  // (the kernels' helpers)
#include "paged_work.h"

namespace nimble {
int fail(int code, const char*, ...) { return code; }
void clear_error() {}
}  // namespace nimble

// ------------------------------------------------------------------------------------------------ calls
using namespace nimble;

static PagedArgs g_args;
static int g_shared[kUnitWords];
constexpr int kRecord = 14;
static int64_t* g_out;
static int64_t g_room, g_count;

static void put_record(const PagedUnit& u, int low, int high, int block0, int block1) {
  if (threadIdx.x != 0) return;
  if (g_count < g_room) {
    const int64_t r[kRecord] = {blockIdx.x, u.s, u.seq.first, u.seq.n, u.seq.length, u.tile, u.head, u.slot, u.parts, u.part, low, high, block0, block1};
    memcpy(g_out + g_count * kRecord, r, sizeof r);
  }
  ++g_count;
}

template <bool CUT>
static void tokens_body() {  // as paged_tokens_kernel goes through its span
  SpanWalk<16, kPagedBlockKeys, CUT> walk(g_args, blockIdx.x);
  walk.clear_item();
  if (walk.none) return;
  for (bool again = true; again; again = CUT && walk.at < walk.end) {
    PagedUnit u;
    u.part = 0;
    int low, high, block0, block1;
    walk.take(u, low, high, block0, block1);
    put_record(u, low, high, block0, block1);
  }
}
static void chunks_body() {  // as paged_chunks_kernel takes its unit
  find_unit<128, 64, 4>(g_args, blockIdx.x, g_shared);
  exchange(0, 5);
  PagedUnit u;
  if (!take_unit(g_args, g_shared, u)) return;
  int low, high, block0, block1;
  unit_keys<128, 64>(g_args, u, low, high, block0, block1);
  put_unit_item(g_args, u);
  put_record(u, low, high, block0, block1);
}

// check_apart of two tensors: 0, or what a refusal returns.
extern "C" int apart(int64_t a, int64_t a_rows, int64_t a_bytes, int64_t a_stride, int64_t b, int64_t b_rows, int64_t b_bytes, int64_t b_stride) {
  return check_apart("", {Extent{"a", (void*)a, a_rows, a_bytes, a_stride}}, {Extent{"b", (void*)b, b_rows, b_bytes, b_stride}});
}

// Workgroups of one call, every `stride`-th from the first on (and all where stride is 1).  out: records of 14 numbers; items: the table that the second
// launch reads, 1 + its workgroups (or more) entries of 12 words, filled by the caller with what an unwritten workspace holds.  Returns the number of records, or
// a negative status.
extern "C" int64_t paged_work(int64_t rows, int64_t count, int64_t width, int64_t heads, int64_t kv_heads, int64_t page, int64_t D, int dtype,
                              int64_t window, const int64_t* offsets, const int64_t* lengths, int64_t stride, int64_t* out, int64_t room, int* items) {
  nimble_paged_plan p;
  const int rc = nimble_paged_attention_plan_of(rows, count, width, heads, kv_heads, page, D, dtype, window, &p);
  if (rc != NIMBLE_OK) return rc;
  const nimble_cache cache{nullptr, nullptr, nullptr, nullptr, 1, kv_heads, page, D, dtype};
  const nimble_sequences seqs{offsets, lengths, nullptr, count, width, rows};
  g_args = PagedArgs{};
  set_extents(g_args, cache, seqs, heads, window);
  set_parts(g_args, p, D, nullptr);
  g_args.items = items;
  g_out = out;
  g_room = room;
  g_count = 0;
  gridDim.x = p.grid;
  for (int64_t w = 0; w < (int64_t)p.grid; w += stride) {
    blockIdx.x = (unsigned)w;
    run_wave(p.kernel == NIMBLE_PAGED_CHUNKS ? chunks_body : p.parts ? tokens_body<true> : tokens_body<false>);
  }
  return g_count;
}
