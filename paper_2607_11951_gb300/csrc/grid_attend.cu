// Attention of a chunk of new tokens over a paged cache (grid_kv_attend).
//
// out = sum_j p_j v_j with p = softmax(scale q k_j) over a token's visible
// positions, in one pass over the keys: a tile of 128 keys gives scores
// S = Q K^T (tensor cores, fp32), each query row keeps its maximum m and sum l
// in fp32, P = exp2((S - m) scale log2 e) is rounded to the cache's type for
// O += P V (tensor cores, fp32), and O and l are rescaled when m grows.
//
// Work.  The query rows of a row b and key head h are its tokens times the
// H / Hk heads that read h (row = token * group + head), so that a key tile is
// read once for all of them.  A unit is 256 such rows, or all of them where
// there are at most 128, with the key tiles they can see.  The tiles of all
// units, one after the other, are cut into equal runs, one per block: a block
// takes the end of one unit, some whole ones and the beginning of another (or
// one key head each, where that is shorter: kJoinCost).  The pieces of a unit
// that was cut are joined by the block that finishes last, in the order of the
// keys whatever the order of the blocks.
//
// A block runs two streams of tiles side by side, each with its scores, output
// rows and four softmax warps, so that the tensor cores work on one stream
// while the other takes its exponentials.  With 256 rows the streams are the
// two halves of the rows and share the key tiles; with up to 128 they take the
// even and the odd tiles of the same rows and are merged at the end.
//
// Roundings: S, m, l and O are fp32.  P is rounded to the cache's type since the
// tensor cores take both operands of a 16-bit product in one type; m may lag
// behind the maximum by 8 exponents (fewer rescalings of O).  In bf16 P is at
// most 2^8, and its relative error of 2^-8 a term is that of the values it
// meets.  In f16 P is 2^7 times as large (at most 2^15, f16 ends below 2^16):
// its relative error is 2^-11 down to 2^-21 of the largest term, below that it
// is held in steps of 2^-24, so that n terms are off by n 2^-32 of the largest
// at most.  l is summed before that rounding; out is rounded once.
//
// Bound by the cached bytes where few rows read many keys: 32 rows of up to 5
// tokens over up to 16,000 (724 MB) take 118 us, 6.1 TB/s; 32 rows of one token
// over up to 2,000 (90 MB) 29 us, of which the start and the joins are some 10;
// one token over 400 takes 9.9.  Bound by the products and the exponentials
// between them where a chunk is long: a call for 2 x 2,000 tokens over 16,000
// (605 GF) takes 454 us, 1,330 TFLOP/s (440 back to back in a graph, 1,370); 27
// prompts of up to 2,000 with 64-wide heads, an exponential for every 256
// operations, 208 us.  The constants' figures below are of 32 + 8 heads of 128
// (prompts: 14 + 2 of 64) in a graph.
#include <dlfcn.h>

#include <cmath>
#include <new>
#include <utility>

#include "grid_kv.cuh"

namespace grid {
namespace {

constexpr int kTile = 128;            // keys of a tile, query rows of a stream
constexpr int kSoftWarps = 8;         // four per stream
constexpr int kLoadWarp = kSoftWarps;      // two that load tiles, of keys and of values,
constexpr int kMmaWarp = kSoftWarps + 2;   // one that multiplies,
constexpr int kQueryWarp = kSoftWarps + 3, kQueryWarps = 1;  // one that loads queries
constexpr int kThreads = (kSoftWarps + 4) * 32;
// A unit's beginning and end cost as much as some tiles (2: 29.1 us for 32 rows of one token, 208 for 27 prompts, 439 for
// 2 x 2,000 tokens over 16,000; 3: 28.8, 214, 442), and runs are not made shorter than a few (3: one token over 2,000 and
// 16,000 takes 12.2 and 24.2 us, 200 tokens over 500 24.7; 5: 15.0, 24.2 and 31.0).  Where every key head can have a block
// of its own and the dearest is no longer than a run and what it costs to join pieces, none is cut (16 rows of one token
// over up to 500: 13.3 -> 11.3 us; one token over 400, 8 + 2 heads of 64: 10.9 -> 9.9).
constexpr int kUnitCost = 2, kMinRun = 3, kJoinCost = 4;
// The costs of all units together, so that places among them are ints.  Rows of an ordered `start` share the tokens of the
// chunk, and what they can cost is checked on the host; rows that overlap, of a start that is not in order, can each be in
// order and cost any multiple of it, which the plan finds (counting in 65,536, less one a warp) before it uses a place.
constexpr int kMostCost = INT32_MAX - (1 << 20);
constexpr int kRing = 8;              // pieces whose bad-page flags are kept at once
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

struct AttendArgs {
  Chunk c;
  const void* q;
  void* out;
  float* lse;
  long long qs[2], os[2];
  int H, Hk, group, sectors;  // sectors: the rows of out begin on 32 bytes
  float scale;
  int32_t* status;
  float4* parts;    // [2 blocks][D / 4][256 rows]
  float2* part_ml;  // [2 blocks][256 rows]: maximum (in exponents of two) and sum (2^kLift times it, as the parts are)
  int* joined;      // [blocks]
  int* gave_up;     // one word: a wait ran out, in this call or an earlier one
};

// ---------------------------------------------------------------------------
// what has no C++ name
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* b, int n) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_at(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_at(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, int bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_at(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* b, int parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(smem_at(b)), "r"(parity)
      : "memory");
  return ok;
}
// Waits for a phase, for two seconds' clocks at most or until another warp
// gave up; false then.  Whole warps wait, and leave together.
__device__ __noinline__ bool bar_wait_long(uint64_t* b, int parity, volatile int* gave_up) {
  const long long t0 = clock64();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 32; ++i)
      if (bar_try(b, parity)) return true;
    if (*gave_up) return false;
    if (clock64() - t0 > 4000000000LL) *gave_up = 1;
  }
}
__device__ __forceinline__ bool bar_wait(uint64_t* b, int parity, volatile int* gave_up) {
  if (__all_sync(~0u, bar_try(b, parity))) return true;
  return __all_sync(~0u, bar_wait_long(b, parity, gave_up));
}
__device__ __forceinline__ bool bar_wait1(uint64_t* b, int parity, volatile int* gave_up) {  // a thread alone
  return bar_try(b, parity) || bar_wait_long(b, parity, gave_up);
}
// One lane of a whole warp, always the same.
__device__ __forceinline__ bool elected() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p;
}
__device__ __forceinline__ void load_tile(const CUtensorMap* m, uint32_t dst, uint64_t* bar, int x, int token, int head,
                                          int page) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
          dst),
      "l"(m), "r"(smem_at(bar)), "r"(x), "r"(token), "r"(head), "r"(page)
      : "memory");
}
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tm_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(b)) : "memory");
}
// D += A B^T, A and B in shared memory, `off` (16-byte units) further on; the
// addition is in here so that it is not made, and kept, ahead of time
template <int kOff>
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile(
      "{\n.reg .pred p;\n.reg .b64 a, b;\nadd.s64 a, %1, %5;\nadd.s64 b, %2, %5;\nsetp.ne.u32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(what), "r"((uint32_t)add), "n"(kOff)
      : "memory");
}
// D += A B, A in tensor memory: step kStep of 16 keys
template <int kStep>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile(
      "{\n.reg .pred p;\n.reg .b32 a;\n.reg .b64 b;\nadd.s32 a, %1, %5;\nadd.s64 b, %2, %6;\nsetp.ne.u32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(what), "r"((uint32_t)add), "n"(kStep * 8), "n"(kStep * 128)
      : "memory");
}
#define O8(x, i) \
  "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define U8(x, i) \
  "+r"(x[i]), "+r"(x[i + 1]), "+r"(x[i + 2]), "+r"(x[i + 3]), "+r"(x[i + 4]), "+r"(x[i + 5]), "+r"(x[i + 6]), "+r"(x[i + 7])
#define I8(x, i) \
  "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
// 32 columns of this thread's row of tensor memory
__device__ __forceinline__ void tm_load32(uint32_t at, uint32_t* x) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : O8(x, 0), O8(x, 8), O8(x, 16), O8(x, 24)
      : "r"(at));
}
__device__ __forceinline__ void tm_load16(uint32_t at, uint32_t* x) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : O8(x, 0), O8(x, 8)
      : "r"(at));
}
__device__ __forceinline__ void tm_store16(uint32_t at, const uint32_t* x) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::I8(
          x, 0),
      I8(x, 8), "r"(at)
      : "memory");
}
// (the registers are named, so that nothing uses them before the wait)
__device__ __forceinline__ void tm_loaded(uint32_t* x) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : U8(x, 0), U8(x, 8), U8(x, 16), U8(x, 24) : : "memory");
}
__device__ __forceinline__ void tm_loaded16(uint32_t* x) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : U8(x, 0), U8(x, 8) : : "memory");
}
__device__ __forceinline__ void tm_loaded16(uint32_t* x, uint32_t* y) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : U8(x, 0), U8(x, 8), U8(y, 0), U8(y, 8) : : "memory");
}
__device__ __forceinline__ void tm_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// P is 2^kLift times the probabilities' numerators.
template <typename T>
constexpr float kLift = std::is_same<T, __half>::value ? 7.f : 0.f;

// 32 keys' probabilities 2^(sc s - base) as pairs of T in the first 16 registers; their sums are added.
template <typename T>
__device__ __forceinline__ void exp32(uint32_t (&x)[32], float sc, float base, Two (&sum)[2]) {
#pragma unroll
  for (int e = 0; e < 32; e += 2) {
    Two a = fma2(Two{__uint_as_float(x[e]), __uint_as_float(x[e + 1])}, sc, -base);
    a = Two{exp2_fast(a.x), exp2_fast(a.y)};
    sum[e / 2 & 1] = add2(sum[e / 2 & 1], a);
    x[e / 2] = pack_of(a.x, a.y, T());
  }
}
__device__ __forceinline__ void max32(const uint32_t (&x)[32], float (&top)[4]) {
#pragma unroll
  for (int e = 0; e < 32; e += 2) top[e / 2 & 3] = max3(top[e / 2 & 3], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
}
__device__ __forceinline__ void hide32(uint32_t (&x)[32], int last) {  // scores past `last` as -inf
  if (last < 31) {
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (e > last) x[e] = 0xFF800000u;
  }
}

// One tile of a row's softmax from nothing: the maximum, base(maximum), then
// the probabilities, from the last keys to the first: they lie (64-wide heads
// apart) over the second half of the scores, which is read before.  Returns their
// sum.  The scores are read from tensor memory twice, the loops are rolled: few
// tiles come here, and those of short calls wait for instructions.
template <typename T, typename Base>
__device__ __forceinline__ float softmax_anew(uint32_t s_at, uint32_t p_at, int last, float sc, Base base) {
  Two sum[2] = {};
  float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  uint32_t x[32];
#pragma unroll 1
  for (int j = 0; j < kTile; j += 32) {
    tm_load32(s_at + j, x);
    tm_loaded(x);
    hide32(x, last - j);
    max32(x, top);
  }
  const float b = base(fmaxf(max3(top[0], top[1], top[2]), top[3]));
#pragma unroll 1
  for (int j = kTile - 32; j >= 0; j -= 32) {
    tm_load32(s_at + j, x);
    tm_loaded(x);
    hide32(x, last - j);
    exp32<T>(x, sc, b, sum);
    tm_store16(p_at + j / 2, x);
  }
  sum[0] = add2(sum[0], sum[1]);
  return sum[0].x + sum[0].y;
}
// The same for many tiles, with loads on their way while the columns before
// are worked on; the last 64 scores are read once.  half() is called once the
// probabilities of the last 64 keys are there.
template <typename T, typename Base, typename Half>
__device__ __forceinline__ float softmax_twice(uint32_t s_at, uint32_t p_at, int last, float sc, Base base, Half half) {
  Two sum[2] = {};
  float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  uint32_t x[32], y[32];
  tm_load32(s_at, x);
  tm_loaded(x);
  tm_load32(s_at + 32, y);
  hide32(x, last);
  max32(x, top);
  tm_loaded(y);
  tm_load32(s_at + 64, x);
  hide32(y, last - 32);
  max32(y, top);
  tm_loaded(x);
  tm_load32(s_at + 96, y);
  hide32(x, last - 64);
  max32(x, top);
  tm_loaded(y);
  hide32(y, last - 96);
  max32(y, top);
  const float b = base(fmaxf(max3(top[0], top[1], top[2]), top[3]));
  exp32<T>(y, sc, b, sum);
  tm_store16(p_at + 48, y);
  tm_load32(s_at + 32, y);
  exp32<T>(x, sc, b, sum);
  tm_store16(p_at + 32, x);
  half();
  tm_loaded(y);
  tm_load32(s_at, x);
  hide32(y, last - 32);
  exp32<T>(y, sc, b, sum);
  tm_store16(p_at + 16, y);
  tm_loaded(x);
  hide32(x, last);
  exp32<T>(x, sc, b, sum);
  tm_store16(p_at, x);
  sum[0] = add2(sum[0], sum[1]);
  return sum[0].x + sum[0].y;
}
// The same in one pass on the maximum b of the tiles before, where the
// probabilities have columns of their own.  `top` gets the tile's own maximum; if
// it turns out to be too far above b, the scores are as they were and the
// result is of no use.
template <typename T>
__device__ __forceinline__ float softmax_once(uint32_t s_at, uint32_t p_at, int last, float sc, float b, float& top) {
  Two sum[2] = {};
  float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  uint32_t x[2][32];
  tm_load32(s_at, x[0]);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t(&y)[32] = x[j & 1];
    tm_loaded(y);
    if (j < 3) tm_load32(s_at + 32 * (j + 1), x[(j + 1) & 1]);
    hide32(y, last - 32 * j);
    max32(y, tops);
    exp32<T>(y, sc, b, sum);
    tm_store16(p_at + 16 * j, y);
  }
  top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]);
  sum[0] = add2(sum[0], sum[1]);
  return sum[0].x + sum[0].y;
}

// Shared memory operand of 128-byte swizzled lines of 64 values: 8 lines are
// 1,024 bytes (the stride); `chunk` is the distance between the column halves
// where the lines run along the output's columns (V), unused where they run
// along the sum (Q, K).
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t chunk) {
  return (uint64_t)((at >> 4) & 0x3FFF) | (uint64_t)((chunk >> 4) & 0x3FFF) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
template <int N, typename F, int... X>
__device__ __forceinline__ void each_step(F f, std::integer_sequence<int, X...>) {
  (f(std::integral_constant<int, X>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each_step(F f) {  // f(0), f(1) .. f(N - 1), the numbers known to the compiler
  each_step<N>(f, std::make_integer_sequence<int, N>());
}
// fp32 accumulators, both operands of type T, 128 rows, n columns; b_rows: B's
// lines run along the columns
template <typename T>
__device__ __forceinline__ uint32_t what_mma(int n, bool b_rows) {
  const uint32_t t = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return 1u << 4 | t << 7 | t << 10 | (b_rows ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | (uint32_t)(kTile / 16) << 24;
}

// ---------------------------------------------------------------------------
// the units of the batch, one after the other
struct Units {
  int b, a, n, len, rows;  // row, its first token, tokens, cached tokens, query rows per key head
  int units, h, qt;        // units per key head; the current one
  int tiles;               // key tiles of the current unit
  int at;                  // where its tiles begin, in costs (kMostCost at most: see there)
};

__device__ __forceinline__ int tiles_of(const Units& u, int group, int qt) {
  if (u.units == 1) return (u.len + u.n + kTile - 1) / kTile;
  const int last = min(u.rows, (qt + 1) * 256) - 1;  // its last query row
  return (u.len + last / group + kTile) / kTile;
}
__device__ __forceinline__ void set_row(const AttendArgs& g, Units& u) {
  u.rows = u.n * g.group;
  u.units = u.rows <= 256 ? 1 : (u.rows + 255) / 256;
}
__device__ __forceinline__ bool open_row(const AttendArgs& g, Units& u, int b) {
  u.b = b;
  if (!row_span(g.c, b, u.a, u.n, u.len) || u.n == 0) return false;
  set_row(g, u);
  return true;
}
// The cost of a key head, by a warp (every lane gets the sum).
__device__ __forceinline__ int head_tiles(const Units& u, int group, int lane) {
  int t = 0;
#pragma unroll 1
  for (int i = lane; i < u.units; i += 32) t += kUnitCost + tiles_of(u, group, i);
  return __reduce_add_sync(~0u, t);
}
__device__ __forceinline__ void next_unit(const AttendArgs& g, Units& u) {
  u.at += u.tiles + kUnitCost;
  if (++u.qt == u.units) {
    u.qt = 0;
    if (++u.h == g.Hk) {
      u.h = 0;
#pragma unroll 1
      while (u.b + 1 < g.c.B && !open_row(g, u, u.b + 1)) {
      }
    }
  }
  u.tiles = tiles_of(u, g.group, u.qt);
}

// All costs cut into runs, one per block, the first `more` of them longer by one.
struct Cut {
  int runs, each, more;
  __device__ __forceinline__ int begin(int i) const { return i * each + min(i, more); }
  __device__ __forceinline__ int run_of(int at) const {
    const int longer = more * (each + 1);
    return at < longer ? at / (each + 1) : more + (at - longer) / each;
  }
};

// One block's part of one unit.
struct Piece {
  bool wide;     // 256 rows: the streams share the tiles; else even and odd tiles
  int t0, t1;    // key tiles
  int n[2];      // tiles of each stream
  int r0;        // first query row
  __device__ __forceinline__ bool ends(const Units& u) const { return u.len + u.n < t1 * kTile; }  // past the row's last token
};
__device__ __forceinline__ Piece piece_of(const Units& u, int lo, int hi) {
  Piece p;
  p.t0 = max(lo, u.at) - u.at;
  p.t1 = min(hi, u.at + u.tiles) - u.at;
  p.wide = u.rows > kTile;
  p.r0 = u.qt * 256;
  const int n = p.t1 - p.t0;
  p.n[0] = p.wide ? n : (n + 1) / 2;
  p.n[1] = p.wide ? (u.rows - p.r0 > kTile ? n : 0) : n / 2;
  return p;
}

template <int D>
struct Layout {
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kStages = D == 128 ? 5 : 10;
  static constexpr int kTiles = 2 * kTileBytes + kStages * kTileBytes;
  static constexpr uint32_t kS = 0, kO = 256;                 // columns of tensor memory: scores, outputs,
  static constexpr uint32_t kP = D == 128 ? 64 : 256 + 2 * D;  // probabilities (over the scores where all columns are taken)
  static constexpr bool kApart = D == 64;                     // probabilities have columns of their own
  static constexpr uint32_t kPStep = D == 128 ? 128 : 64;
};

struct Shared {
  uint64_t full[10], empty[10];
  uint64_t q_ready[2], q_free[2], s_ready[2], p_half[2], p_ready[2], o_ready[2], all;
  float2 ml[2][kTile];
  Units units[kSoftWarps];
  int4 sums[kThreads / 32];  // of the warps: cost, rows, dearest row, cost in 65,536
  int first, per, row[4], gave_up, last, broken, crowded, bad[2][kRing];
  uint32_t tmem;
};

constexpr int kSharedRoom = 3 << 10;  // in front of the tiles, which begin on 1,024 bytes

template <int D>
constexpr size_t smem_bytes() {
  static_assert(sizeof(Shared) <= kSharedRoom);
  return kSharedRoom + Layout<D>::kTiles;
}

// A block that gave up sets the handle's word, then writes GRID_ST_BOUND to all rows.
__device__ __noinline__ void report_bound(int* gave_up, int32_t* status, int B) {
  if (threadIdx.x == 0) {
    atomicExch(gave_up, 1);
    __threadfence();
  }
  __syncthreads();
  for (int b = threadIdx.x; b < B; b += kThreads) status[b] = GRID_ST_BOUND;
}
// By a warp that stored its rows' status: what it stored before a block set the word is overwritten by that block, what it
// stored after it sees the word.
__device__ __noinline__ void report_again(int* gave_up, int32_t* status, int B) {
  __threadfence();
  if (__ldcg(gave_up) && threadIdx.x % 32 == 0)
    for (int b = blockIdx.x; b < B; b += gridDim.x) status[b] = GRID_ST_BOUND;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
    k_attend(const AttendArgs g, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using L = Layout<D>;
  extern __shared__ __align__(1024) uint8_t raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  uint8_t* tiles = raw + kSharedRoom;
  const uint32_t q_at = smem_at(tiles), ring = q_at + 2 * L::kTileBytes;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Chunk& c = g.c;
  if (warp == kLoadWarp && lane < 2)
    asm volatile("prefetch.tensormap [%0];" ::"l"(lane ? &v_map : &k_map) : "memory");
  if (tid == 0) {
    for (int i = 0; i < L::kStages; ++i) {
      bar_init(&sh.full[i], 1);
      bar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(&sh.q_ready[i], kQueryWarps);
      bar_init(&sh.q_free[i], 1);
      bar_init(&sh.s_ready[i], 1);
      bar_init(&sh.p_half[i], 4);
      bar_init(&sh.p_ready[i], 4);
      bar_init(&sh.o_ready[i], 1);
    }
    bar_init(&sh.all, kSoftWarps);
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_at(&sh.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tm_before();
  }
  pdl_wait();

  const int broken = tid == 0 ? __ldcg(g.gave_up) : 0;
  // How many tiles there are in all, and the row that this block begins in.
  Cut cut;
  bool whole_heads;
  Units u;
  {
    // A thread's rows are `per` neighbours, one of them at a time; rows of several units go to the warps in turn.
    const int per = (c.B + kThreads - 1) / kThreads;
    int* many = reinterpret_cast<int*>(tiles);  // [kThreads][3]: tokens, cached tokens, cost (the tiles come later)
    auto row_cost = [&](int b) {
      const bool some = b < min(c.B, (tid + 1) * per) && open_row(g, u, b);
      int t = some && u.units == 1 ? kUnitCost + tiles_of(u, g.group, 0) : 0, at = -1;
      if (tid == 0) sh.last = 0;
      if (!__syncthreads_or(some && u.units > 1)) return t;
      if (some && u.units > 1) {
        at = atomicAdd(&sh.last, 1);
        many[3 * at] = u.n, many[3 * at + 1] = u.len;
      }
      __syncthreads();
#pragma unroll 1
      for (int i = warp; i < sh.last; i += kThreads / 32) {
        Units v;
        v.n = many[3 * i], v.len = many[3 * i + 1];
        set_row(g, v);
        const int sum = head_tiles(v, g.group, lane);
        if (lane == 0) many[3 * i + 2] = sum;
      }
      __syncthreads();
      return at >= 0 ? many[3 * at + 2] : t;
    };
    int mine = 0, rows = 0, most = 0, t = 0;  // of this thread: their cost, how many have tokens, the dearest
    unsigned high = 0, low = 0;               // the cost in halves, which no 65,535 rows overflow
#pragma unroll 1
    for (int i = 0; i < per; ++i) {
      t = row_cost(tid * per + i);
      mine += t * g.Hk, rows += t > 0, most = max(most, t);
      high += (unsigned)(t * g.Hk) >> 16, low += (unsigned)(t * g.Hk) & 0xFFFFu;
    }
    auto up_to = [&](int x) {  // the sum over the lanes up to this one
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
      }
      return x;
    };
    int pre = up_to(mine), pre_rows = up_to(rows);
    most = __reduce_max_sync(~0u, most);
    high = __reduce_add_sync(~0u, high) + (__reduce_add_sync(~0u, low) >> 16);
    if (lane == 31) sh.sums[warp] = make_int4(pre, pre_rows, most, (int)high);
    __syncthreads();
    int total = 0, all_rows = 0, coarse = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
      const int4 x = sh.sums[w];
      if (w < warp) pre += x.x, pre_rows += x.y;
      total += x.x, all_rows += x.y, most = max(most, x.z), coarse += x.w;
    }
    const bool crowded = coarse > (kMostCost >> 16);
    if (tid == 0) sh.crowded = crowded;
    pre -= mine, pre_rows -= rows;
    cut.runs = crowded ? 0 : min((int)gridDim.x, (total + kMinRun - 1) / kMinRun);
    cut.each = cut.runs ? total / cut.runs : 0;
    // A key head to a block, where that makes no block's work longer than a run and what joining takes.
    whole_heads = !crowded && all_rows <= (int)gridDim.x / g.Hk && most <= cut.each + kJoinCost;
    if (whole_heads) cut.runs = all_rows * g.Hk, pre = pre_rows * g.Hk, mine = rows * g.Hk;
    cut.each = cut.runs ? total / cut.runs : 0;
    cut.more = total - cut.runs * cut.each;
    const int lo = whole_heads ? (int)blockIdx.x : cut.begin(blockIdx.x);
    const bool here = (int)blockIdx.x < cut.runs && pre <= lo && lo < pre + mine;
#pragma unroll 1
    for (int i = 0; i < per; ++i) {
      if (per > 1) t = row_cost(tid * per + i);
      const int each = whole_heads ? t > 0 : t;
      if (here && pre <= lo && lo < pre + each * g.Hk) {
        sh.row[0] = u.b, sh.row[1] = u.a, sh.row[2] = u.n, sh.row[3] = u.len;
        sh.first = pre;
        sh.per = t;
      }
      pre += each * g.Hk;
    }
  }
  if (tid == 0) sh.broken = broken;
  __syncthreads();
  // (Where a call gave up, units may wait for pieces that never came: this one does nothing but report it.)
  const bool works = (int)blockIdx.x < cut.runs && !sh.broken;
  tm_after();
  const uint32_t tmem = sh.tmem;
  const int lo = !works || whole_heads ? 0 : cut.begin(blockIdx.x), hi = !works ? 0 : whole_heads ? sh.per : cut.begin(blockIdx.x + 1);
  volatile int* gave_up = &sh.gave_up;
  if (works) {  // the unit that the run begins in
    u.b = sh.row[0], u.a = sh.row[1], u.n = sh.row[2], u.len = sh.row[3];
    set_row(g, u);
    u.h = whole_heads ? (int)blockIdx.x - sh.first : (lo - sh.first) / sh.per;
    u.at = whole_heads ? 0 : sh.first + u.h * sh.per;
    u.qt = 0;
    if (u.units == 1) {
      u.tiles = tiles_of(u, g.group, 0);
      u.at += kUnitCost;
    } else
#pragma unroll 1
    for (int i = 0;; i += 32) {  // 32 units at once
      const int mine = i + lane < u.units ? kUnitCost + tiles_of(u, g.group, i + lane) : 0;
      int sum = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += x;
      }
      const unsigned past = __ballot_sync(~0u, lo < u.at + sum);
      if (past || i + 32 >= u.units) {
        const int l = past ? __ffs(past) - 1 : 0;
        u.qt = i + l;
        u.tiles = __shfl_sync(~0u, mine, l) - kUnitCost;
        u.at += __shfl_sync(~0u, sum - mine, l) + kUnitCost;
        break;
      }
      u.at += __shfl_sync(~0u, sum, 31);
    }
  }

  if (warp < kMmaWarp && warp >= kLoadWarp) {
    // ---- two warps keep the ring of tiles full, one with keys and one with values: a lane per page and half of the
    // columns (a copy takes its lane about 90 cycles to issue, and pages of 16 tokens make 16 copies of a tile)
    async_fence();  // (the plan was made where the tiles come)
    const bool v = warp != kLoadWarp;
    int base = 0, it = 0;  // the piece's first item of the ring, and this warp's
    if (works) {
      const int box = min(kTile, 1 << c.log_page), pages = kTile / box, boxes = pages * (D / 64);
      const int part = lane / pages, page_lane = lane - part * pages;
      const uint32_t to = ring + part * (kTile * 128) + page_lane * box * 128;
      const CUtensorMap* map = v ? &v_map : &k_map;
      bool ok = true;
      // the ids of 32 pages at a time, the lane's its own: those of the tile, and those after them
      int row = -1, block = 0, id = 0, id_next = 0;
#pragma unroll 1
      for (int k = 0; ok && u.at < hi; ++k) {
        const Piece p = piece_of(u, lo, hi);
        const int used = (u.len + u.n + (1 << c.log_page) - 1) >> c.log_page;  // pages of the row
        int* bad = &sh.bad[v][k % kRing];
        if (lane == 0) *bad = 0;
        __syncwarp();
        auto fetch = [&](int bl) {  // -1: outside the cache; past the row: one past the pool, which loads zeros
          const int pg = bl * 32 + lane;
          return pg < used ? page_of(c, u.b, pg << c.log_page) : c.n_pages;
        };
        const int n = p.t1 - p.t0;
#pragma unroll 1
        for (int j = 0; j < n; ++j) {
          // its place in the order in which the products take them: K0 V0 K1 V1 ... where the streams share the tiles,
          // K0 K1 V0 K2 V1 K3 ... where they take them in turn
          it = base + (p.wide ? 2 * j + v : v ? min(2 * j + 2, 2 * n - 1) : max(j, 2 * j - 1));
          const int st = it % L::kStages, token = (p.t0 + j) * kTile, pg = token >> c.log_page;
          if (row != u.b || pg >> 5 != block) {
            id = row == u.b && pg >> 5 == block + 1 ? id_next : fetch(pg >> 5);
            row = u.b;
            block = pg >> 5;
            id_next = fetch(block + 1);
          }
          int page = __shfl_sync(~0u, id, (pg + page_lane) & 31);
          if (page < 0) {
            page = c.n_pages;
            if (lane < boxes) *bad = 1;
          }
          if (!(ok = bar_wait(&sh.empty[st], ((it / L::kStages) & 1) ^ 1, gave_up))) break;
          if (lane == 0) bar_expect(&sh.full[st], L::kTileBytes);
          __syncwarp();
          if (lane < boxes)
            load_tile(map, to + st * L::kTileBytes, &sh.full[st], part * 64, token & ((1 << c.log_page) - 1), u.h, page);
        }
        base += 2 * n;
        next_unit(g, u);
      }
    }
    // ---- then one of them reports the rows, and zeros those that are not in order
    for (int b = blockIdx.x; !v && b < c.B; b += gridDim.x) {
      int a, n, len;
      const bool ordered = row_span(c, b, a, n, len) && !sh.crowded;
      bool good = ordered;
      if (good && n)
        for (int p = lane; p <= (len + n - 1) >> c.log_page; p += 32) good = good && page_of(c, b, p << c.log_page) >= 0;
      good = __all_sync(~0u, good);
      if (lane == 0) g.status[b] = good ? GRID_ST_OK : GRID_ST_PAGES;
      if (!ordered) {
        const int from = max(0, a), to = (int)min((long long)c.N, (long long)a + n);
        for (long long i = (long long)from * g.H; i < (long long)to * g.H; ++i) {
          const long long tok = i / g.H, h = i % g.H;
          for (int x = lane; x < D / 8; x += 32)
            *reinterpret_cast<uint4*>((T*)g.out + tok * g.os[0] + h * g.os[1] + x * 8) = make_uint4(0, 0, 0, 0);
          if (g.lse && lane == 0) g.lse[i] = -INFINITY;
        }
      }
    }
    if (!v) report_again(g.gave_up, g.status, c.B);
    // (No copy is in flight when the block ends: every tile was waited for.  Where a wait was given up, what is still on
    // its way has a tenth of a millisecond to land.)
    if (*gave_up)
      for (const long long t0 = clock64(); clock64() - t0 < 200000;) {
      }
  } else if (warp == kMmaWarp) {
    // ---- one thread issues the products, with as little as can be between them
    if (works && elected()) {
      const uint32_t what_qk = what_mma<T>(kTile, false), what_pv = what_mma<T>(D, true);
      int st = 0, ph = 0;               // the next item of the ring and its phase
      int n_q[2] = {0, 0}, n_p[2] = {0, 0}, n_h[2] = {0, 0};
      auto step = [&](int& a, int& b) {
        if (++a == L::kStages) a = 0, b ^= 1;
      };
      auto qk = [&](int s, bool first, bool last, int at, int phase, bool release) {
        if (first && !bar_wait1(&sh.q_ready[s], n_q[s]++ & 1, gave_up)) return false;
        if (!bar_wait1(&sh.full[at], phase, gave_up)) return false;
        tm_after();
        const uint32_t a = q_at + s * L::kTileBytes, b = ring + at * L::kTileBytes;
        const uint64_t da = operand(a, 16), db = operand(b, 16);
        each_step<D / 16>([&](auto x) {
          constexpr int kX = decltype(x)::value;
          mma_ss<(kX / 4) * (kTile * 128 / 16) + (kX % 4) * 2>(tmem + L::kS + s * 128, da, db, what_qk, kX > 0);
        });
        tm_commit(&sh.s_ready[s]);
        if (release) tm_commit(&sh.empty[at]);
        if (last) tm_commit(&sh.q_free[s]);
        return true;
      };
      auto pv = [&](int s, bool first, bool last, int at, int phase, bool release, bool halves) {
        if (!bar_wait1(&sh.full[at], phase, gave_up)) return false;
        // (a wide piece's product begins with the second half of the probabilities, which is there first)
        if (halves ? !bar_wait1(&sh.p_half[s], n_h[s]++ & 1, gave_up) : !bar_wait1(&sh.p_ready[s], n_p[s]++ & 1, gave_up)) return false;
        tm_after();
        const uint32_t b = ring + at * L::kTileBytes;
        const uint64_t db = operand(b, kTile * 128);
        constexpr int kHalf = kTile / 32;
        const uint32_t d = tmem + L::kO + s * D, pr = tmem + L::kP + s * L::kPStep;
        each_step<kHalf>([&](auto x) {
          constexpr int kX = decltype(x)::value;
          mma_ts<kHalf + kX>(d, pr, db, what_pv, !first || kX > 0);
        });
        if (halves) {
          if (!bar_wait1(&sh.p_ready[s], n_p[s]++ & 1, gave_up)) return false;
          tm_after();
        }
        each_step<kHalf>([&](auto x) { mma_ts<decltype(x)::value>(d, pr, db, what_pv, true); });
        if (last) tm_commit(&sh.o_ready[s]);
        if (release) tm_commit(&sh.empty[at]);
        return true;
      };
      bool ok = true;
#pragma unroll 1
      while (ok && u.at < hi) {
        const Piece p = piece_of(u, lo, hi);
        if (p.wide) {
          const int n = p.n[0];
          const bool both = p.n[1] > 0;
          ok = qk(0, true, n == 1, st, ph, !both) && (!both || qk(1, true, n == 1, st, ph, true));
#pragma unroll 1
          for (int i = 0; ok && i < n; ++i) {
            step(st, ph);
            const int v = st, vp = ph;
            step(st, ph);
            const bool last = i + 1 == n;
            ok = pv(0, i == 0, last, v, vp, !both, !L::kApart) && (last || qk(0, false, i + 2 == n, st, ph, !both));
            if (ok && both) ok = pv(1, i == 0, last, v, vp, true, !L::kApart) && (last || qk(1, false, i + 2 == n, st, ph, true));
          }
        } else {
          const int n = p.t1 - p.t0;
#pragma unroll 1
          for (int x = -2; ok && x < 2 * n; ++x) {  // K0 K1 V0 K2 V1 K3 ..., the even tiles to stream 0, the odd ones to 1
            const bool v = x >= 0 && !(x & 1);
            const int t = x < 0 ? x + 2 : x / 2 + (v ? 0 : 2);
            if (t >= n) continue;
            ok = v ? pv(t & 1, t < 2, t + 2 >= n, st, ph, true, false)
                   : qk(t & 1, t < 2, t + 2 >= n, st, ph, true);
            step(st, ph);
          }
        }
        next_unit(g, u);
      }
    }
    __syncwarp();
  } else if (warp >= kQueryWarp) {
    // ---- one warp brings the next unit's queries as soon as the last product has read the ones before
    constexpr int kPer = D / 16, kRows = 16;  // a row's 16-byte parts, half of them to each of two lanes
    const int part = lane % 2 * kPer, step_head = kRows % g.group;
    const long long step_src = kRows / g.group * g.qs[0] + step_head * g.qs[1];  // (where the head does not pass its group's end)
    int n_f[2] = {0, 0};
    bool ok = works;
#pragma unroll 1
    while (ok && u.at < hi) {
      const Piece p = piece_of(u, lo, hi);
#pragma unroll 1
      for (int s = 0; ok && s < 2; ++s) {
        if (!p.n[s]) continue;
        ok = bar_wait(&sh.q_free[s], (n_f[s]++ & 1) ^ 1, gave_up);
        if (!ok) break;
        const int r0 = p.r0 + (p.wide ? s * kTile : 0), rows = min(kTile, u.rows - r0);
        // (rows past the unit's last are left as they are: they have no part in any other row)
        const int r_first = lane / 2, row = r0 + r_first, t = row / g.group;
        int of = row - t * g.group;  // the query head within its group
        const T* src = (const T*)g.q + (long long)(u.a + t) * g.qs[0] + (long long)(u.h * g.group + of) * g.qs[1] + part * 8;
        const uint32_t to = q_at + s * L::kTileBytes;
#pragma unroll 1
        for (int r = r_first; r < rows; r += kRows) {
#pragma unroll
          for (int x = 0; x < kPer; ++x) {
            const int y = part + x;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + r * 128 + (y / 8) * (kTile * 128) + ((y % 8) ^ (r & 7)) * 16),
                         "l"(src + x * 8)
                         : "memory");
          }
          of += step_head;
          src += step_src;
          if (of >= g.group) {
            of -= g.group;
            src += g.qs[0] - g.group * g.qs[1];
          }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        async_fence();
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.q_ready[s]);
      }
      next_unit(g, u);
    }
  } else if (works) {
    // ---- eight warps: softmax of the tiles, rows out
    // (the warp's unit lies in shared memory: registers are short)
    Units& w = sh.units[warp];
    if (lane == 0) w = u;
    __syncwarp();
    const int s = warp / 4, r = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // (32 lanes of tensor memory, in the upper half of an address)
    const uint32_t s_at = tmem + lanes + L::kS + s * 128, p_at = tmem + lanes + L::kP + s * L::kPStep;
    const uint32_t o_at = tmem + lanes + L::kO;
    const float sc = g.scale * kLog2e;
    int n_s = 0, n_o[2] = {0, 0}, n_all = 0, items = 0;
    auto sync_all = [&]() {
      __syncwarp();
      if (lane == 0) bar_arrive(&sh.all);
      return bar_wait(&sh.all, n_all++ & 1, gave_up);
    };
    bool ok = true;
    for (int k = 0; ok && w.at < hi; ++k) {
      const Piece p = piece_of(w, lo, hi);
      const int row = p.r0 + r + (p.wide ? s * kTile : 0);
      const bool live = row < w.rows;
      const bool warp_live = __any_sync(~0u, live);
      const int t = live ? row / g.group : w.n - 1, head = live ? w.h * g.group + row - t * g.group : 0;
      const int sees = w.len + t;  // the last position that the row's token sees
      items += 2 * (p.t1 - p.t0);    // of the ring, up to the piece's end
      float m = -INFINITY, l = 0.f;  // the maximum is scaled: in exponents of two
      for (int i = 0; i < p.n[s]; ++i) {
        if (!bar_wait(&sh.s_ready[s], n_s++ & 1, gave_up)) {
          ok = false;
          break;
        }
        if (i + 1 == p.n[s] && p.ends(w) && (p.wide ? s == 0 : ((p.t1 - p.t0 - 1) & 1) == s)) {
          // values past the row's last token are not the row's, and 0 times their bits may be NaN: zeros in their place
          // (the ring's place of the piece's last values cannot be taken again before their product)
          const int st = (items - 1) % L::kStages, rows = w.len + w.n - (p.t1 - 1) * kTile;
          ok = bar_wait(&sh.full[st], ((items - 1) / L::kStages) & 1, gave_up);
          if (!ok) break;
          for (int y = rows * 8 + r; y < kTile * 8; y += kTile)
            for (int half = 0; half < D / 64; ++half)
              *reinterpret_cast<uint4*>(tiles + (2 + st) * L::kTileBytes + half * (kTile * 128) + y * 16) = make_uint4(0, 0, 0, 0);
          async_fence();
        }
        if (warp_live) {
          tm_after();
          const int tile = p.wide ? p.t0 + i : p.t0 + 2 * i + s;
          const int last = sees - tile * kTile;  // the tile's last visible key
          auto base = [&](float top) {
            const float now = top * sc;
            // The maximum is moved only where it grew by more than 8 (the probabilities stay below 2^8, or 2^15 in
            // f16, and lose nothing in floating point): few tiles rescale what came before them.
            if (__any_sync(~0u, live && now - m > 8.f)) {
              const float most = fmaxf(m, now), f = m > -INFINITY ? exp2_fast(m - most) : 0.f;
              if (i > 0) {
#pragma unroll 1
                for (int j = 0; j < D; j += 16) {
                  uint32_t o[16];
                  tm_load16(o_at + s * D + j, o);
                  tm_loaded16(o);
#pragma unroll
                  for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                  tm_store16(o_at + s * D + j, o);
                }
              }
              l *= f;
              m = most;
            }
            return (m > -INFINITY ? m : 0.f) - kLift<T>;
          };
          float added, top;  // (the base may rescale l first)
          if constexpr (L::kApart) {
            bool fits = false;
            if (p.wide && i > 0) {
              added = softmax_once<T>(s_at, p_at, last, sc, (m > -INFINITY ? m : 0.f) - kLift<T>, top);
              fits = !__any_sync(~0u, live && top * sc - m > 8.f);
            }
            if (!fits) added = softmax_anew<T>(s_at, p_at, last, sc, base);
          } else {
            added = p.wide ? softmax_twice<T>(s_at, p_at, last, sc, base,
                                              [&]() {
                                                tm_stored();
                                                tm_before();
                                                __syncwarp();
                                                if (lane == 0) bar_arrive(&sh.p_half[s]);
                                              })
                           : softmax_anew<T>(s_at, p_at, last, sc, base);
          }
          l += added;
          tm_stored();
          tm_before();
        } else if (!L::kApart && p.wide) {
          if (lane == 0) bar_arrive(&sh.p_half[s]);
        }
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.p_ready[s]);
      }
      if (!ok) break;
      // ---- the rows' outcome
      const bool whole = p.t0 == 0 && p.t1 == w.tiles;
      const int c0 = cut.run_of(w.at);
      const int slot = 2 * blockIdx.x + ((int)blockIdx.x == c0 ? 1 : 0);
      float4* part = g.parts + (size_t)slot * (D / 4) * 256;
      T* dst = (T*)g.out + (long long)(w.a + t) * g.os[0] + (long long)head * g.os[1];
      float f[2];
      if (!p.wide) {  // both streams hold the same rows: each of the two halves of the warps takes half of the columns
        sh.ml[s][r] = make_float2(m, l);
        if (!sync_all()) break;
        const float2 x = sh.ml[0][r], y = sh.ml[1][r];
        m = fmaxf(x.x, y.x);
        f[0] = x.x > -INFINITY ? exp2_fast(x.x - m) : 0.f;
        f[1] = y.x > -INFINITY ? exp2_fast(y.x - m) : 0.f;
        l = x.y * f[0] + y.y * f[1];
      } else {
        f[0] = f[1] = 1.f;
      }
      for (int z = 0; z < 2 && ok; ++z)
        if (p.n[z]) {
          if (!p.wide || z == s) ok = bar_wait(&sh.o_ready[z], n_o[z] & 1, gave_up);
          ++n_o[z];
        }
      if (!ok) break;
      // A sum below zero: some key that the rows may read is in no page of the cache (known once all tiles were), and they
      // get zeros.  A sum that is no number, of a query that is none, gives NaN.
      if (sh.bad[0][k % kRing] | sh.bad[1][k % kRing]) l = -1.f;
      if (warp_live) {
        tm_after();
        const float by = !whole ? 1.f : __frcp_rn(l), f0 = f[0] * by, f1 = f[1] * by;
        const bool two = !p.wide && p.n[1];
        const int from = p.wide ? 0 : s * (D / 2), to = p.wide ? D : from + D / 2;
        const int part_row = r + (p.wide ? s * kTile : 0);
#pragma unroll 1
        for (int j = from; j < to; j += 16) {
          uint32_t o[16], o1[16] = {};
          tm_load16(o_at + (p.wide ? s * D : 0) + j, o);
          if (two) tm_load16(o_at + D + j, o1);
          tm_loaded16(o, o1);
          float y[16];
          if (two) {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = fmaf(__uint_as_float(o1[e]), f1, __uint_as_float(o[e]) * f0);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = __uint_as_float(o[e]) * f0;
          }
          if (live && whole) {
            const uint4 none = {}, a = l < 0.f ? none : pack8<T>(y), b = l < 0.f ? none : pack8<T>(y + 8);
            if (g.sectors) {
              asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + j), "r"(a.x), "r"(a.y), "r"(a.z),
                           "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                           : "memory");
            } else {
              *reinterpret_cast<uint4*>(dst + j) = a;
              *reinterpret_cast<uint4*>(dst + j + 8) = b;
            }
          } else if (live) {
#pragma unroll
            for (int e = 0; e < 16; e += 4)
              __stcg(part + (size_t)((j + e) / 4) * 256 + part_row, make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]));
          }
          __syncwarp();
        }
        if (live && (p.wide || s == 0)) {
          if (whole) {
            if (g.lse) g.lse[(long long)(w.a + t) * g.H + head] = l < 0.f ? -INFINITY : (m - kLift<T> + log2f(l)) * kLn2;
          } else {
            __stcg(g.part_ml + (size_t)slot * 256 + part_row, make_float2(m, l));
          }
        }
        tm_before();
      }
      if (!whole) {
        // ---- the last block of the unit joins its pieces
        const int c1 = cut.run_of(w.at + w.tiles - 1);
        if (!sync_all()) break;
        if (tid == 0) {
          int n;  // (after the barrier: releases what all the others wrote, too)
          asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(n) : "l"(&g.joined[c0]) : "memory");
          sh.last = n == c1 - c0;
          if (sh.last) g.joined[c0] = 0;
        }
        if (!sync_all()) break;
        if (sh.last) {
          const int rows = min(256, w.rows - p.r0);
          int cols = 8;  // of a row to a thread: all of them where there are rows enough
          while (cols < D && rows * (D / cols) > kSoftWarps * 32) cols *= 2;
          for (int x = tid; x < rows * (D / cols); x += kSoftWarps * 32) {
            const int rr = x % rows, from = x / rows * cols;
            const int qrow = p.r0 + rr, tok = qrow / g.group, hh = w.h * g.group + qrow - tok * g.group;
            T* to = (T*)g.out + (long long)(w.a + tok) * g.os[0] + (long long)hh * g.os[1];
            // So many columns of so many pieces at a time, the sums rescaled as they go: no load of a round waits for another
            // (16 columns at most instead of 32: 27 prompts 212 us instead of 208; three pieces of 32 columns instead of two: 2 x
            // 2,000 tokens over 16,000 450 instead of 443; two of 8 columns instead of six: one token over 16,000 with 16 query
            // heads and one key head 18.7 instead of 17.1).
            auto add_up = [&](auto columns, auto pieces, int j) {
              constexpr int kN = decltype(columns)::value, kP = decltype(pieces)::value;
              float acc[kN] = {}, most = -INFINITY, z = 0.f;
              bool bad = false;
#pragma unroll 1
              for (int b = c0; b <= c1; b += kP) {
                float2 e[kP];
                float4 v[kP][kN / 4];
#pragma unroll
                for (int y = 0; y < kP; ++y) {
                  const int piece = min(b + y, c1);
                  const size_t slot = 2 * piece + (piece == c0);
                  e[y] = __ldcg(g.part_ml + slot * 256 + rr);
#pragma unroll
                  for (int x = 0; x < kN / 4; ++x) v[y][x] = __ldcg(g.parts + (slot * (D / 4) + j / 4 + x) * 256 + rr);
                }
                float now = most;
#pragma unroll
                for (int y = 0; y < kP; ++y) {
                  if (b + y > c1) e[y] = make_float2(-INFINITY, 0.f);  // (past the last)
                  now = fmaxf(now, e[y].x);
                  bad |= e[y].y < 0.f;
                }
                const float base = now > -INFINITY ? now : 0.f, f = exp2_fast(most - base);
                most = now;
                z *= f;
#pragma unroll
                for (int x = 0; x < kN; ++x) acc[x] *= f;
#pragma unroll
                for (int y = 0; y < kP; ++y) {
                  const float fy = exp2_fast(e[y].x - base);
                  z = fmaf(e[y].y, fy, z);
#pragma unroll
                  for (int x = 0; x < kN / 4; ++x) {
                    acc[4 * x] = fmaf(v[y][x].x, fy, acc[4 * x]);
                    acc[4 * x + 1] = fmaf(v[y][x].y, fy, acc[4 * x + 1]);
                    acc[4 * x + 2] = fmaf(v[y][x].z, fy, acc[4 * x + 2]);
                    acc[4 * x + 3] = fmaf(v[y][x].w, fy, acc[4 * x + 3]);
                  }
                }
              }
              const float by = __frcp_rn(z);
#pragma unroll
              for (int e = 0; e < kN; ++e) acc[e] = bad ? 0.f : acc[e] * by;
#pragma unroll
              for (int e = 0; e < kN; e += 8) *reinterpret_cast<uint4*>(to + j + e) = pack8<T>(acc + e);
              if (g.lse && j == 0) g.lse[(long long)(w.a + tok) * g.H + hh] = bad ? -INFINITY : (most - kLift<T> + log2f(z)) * kLn2;
            };
            if (cols >= 32)
#pragma unroll 1
              for (int j = from; j < from + cols; j += 32) add_up(std::integral_constant<int, 32>(), std::integral_constant<int, 2>(), j);
            else
#pragma unroll 1
              for (int j = from; j < from + cols; j += 8) add_up(std::integral_constant<int, 8>(), std::integral_constant<int, 6>(), j);
          }
        }
      } else if (!p.wide) {
        ok = sync_all();  // both halves have read both streams' rows before the next piece writes them
      }
      __syncwarp();
      if (lane == 0) next_unit(g, w);
      __syncwarp();
    }
    if (!ok) *gave_up = 1;
  }
  __syncthreads();
  if (sh.gave_up) report_bound(g.gave_up, g.status, c.B);
  if (warp == kMmaWarp) {
    tm_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// A pool as a tensor map: boxes of 64 values of up to 128 tokens of one head of
// one page.  The encoder is the driver library's, which the CUDA runtime has loaded.
int make_map(const grid_kv_pages& p, void* pool, const int64_t* stride, CUtensorMap* map) {
  static const auto encode = reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>([]() -> void* {
    void* lib = dlopen("libcuda.so.1", RTLD_LAZY);
    return lib ? dlsym(lib, "cuTensorMapEncodeTiled") : nullptr;
  }());
  if (!encode) return set_error(GRID_E_CUDA, "grid_kv_create: no CUDA driver library");
  const cuuint64_t dim[4] = {(cuuint64_t)p.head_dim, (cuuint64_t)p.page_size, (cuuint64_t)p.n_kv_heads, (cuuint64_t)p.n_pages};
  const cuuint64_t step[3] = {(cuuint64_t)stride[1] * 2, (cuuint64_t)stride[2] * 2, (cuuint64_t)stride[0] * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)std::min(p.page_size, kTile), 1, 1}, one[4] = {1, 1, 1, 1};
  const CUresult r = encode(map, p.dtype == GRID_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                            4, pool, dim, step, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS)
    return set_error(GRID_E_INVALID_ARG, "grid_kv_create: the pools' strides make no tensor map (" + std::to_string((int)r) + ")");
  return GRID_OK;
}

template <typename F>
cudaError_t each_kernel(F f) {
  cudaError_t e;
  if ((e = f(k_attend<__nv_bfloat16, 64>, smem_bytes<64>())) || (e = f(k_attend<__nv_bfloat16, 128>, smem_bytes<128>())) ||
      (e = f(k_attend<__half, 64>, smem_bytes<64>())))
    return e;
  return f(k_attend<__half, 128>, smem_bytes<128>());
}

}  // namespace
}  // namespace grid

using namespace grid;

extern "C" int grid_kv_create(const grid_kv_pages* p, grid_kv** out) {
  if (!p || !out || !p->d_k || !p->d_v || (uintptr_t)p->d_k % 16 || (uintptr_t)p->d_v % 16 || p->n_pages <= 0 ||
      p->n_heads <= 0 || p->n_kv_heads <= 0 || p->n_heads % p->n_kv_heads)
    return set_error(GRID_E_INVALID_ARG, "grid_kv_create: bad arguments");
  if (p->dtype != GRID_DTYPE_BF16 && p->dtype != GRID_DTYPE_F16)
    return set_error(GRID_E_INVALID_ARG, "grid_kv_create: a cache is of bf16 or f16");
  if (p->head_dim != 64 && p->head_dim != 128)
    return set_error(GRID_E_INVALID_ARG, "grid_kv_create: heads of 64 or 128 values");
  if (p->page_size < 8 || p->page_size > 1024 || (p->page_size & (p->page_size - 1)))
    return set_error(GRID_E_INVALID_ARG, "grid_kv_create: page_size is a power of two in 8 .. 1024");
  for (int i = 0; i < 3; ++i)
    if (p->k_stride[i] <= 0 || p->v_stride[i] <= 0 || p->k_stride[i] % 8 || p->v_stride[i] % 8)
      return set_error(GRID_E_INVALID_ARG, "grid_kv_create: strides are positive multiples of 8 elements");
  grid_kv* kv = new (std::nothrow) grid_kv;
  if (!kv) return set_error(GRID_E_TOO_LARGE, "grid_kv_create: out of host memory");
  kv->p = *p;
  while (1 << kv->log_page < p->page_size) ++kv->log_page;
  int rc = make_map(*p, p->d_k, p->k_stride, &kv->k_map), dev = 0;
  if (!rc) rc = make_map(*p, p->d_v, p->v_stride, &kv->v_map);
  cudaError_t e = cudaSuccess;
  if (!rc && (e = cudaGetDevice(&dev)) == cudaSuccess &&
      (e = cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, dev)) == cudaSuccess) {
    const size_t slots = 2 * (size_t)kv->sms * 256;
    if (!(rc = kv->mem.alloc(slots * p->head_dim * 4, (void**)&kv->parts)) &&
        !(rc = kv->mem.alloc(slots * sizeof(float2), (void**)&kv->part_ml)) &&
        !(rc = kv->mem.alloc(kv->sms * sizeof(int), (void**)&kv->joined)) &&
        !(rc = kv->mem.alloc(sizeof(int), (void**)&kv->gave_up)) &&
        (e = cudaMemset(kv->joined, 0, kv->sms * sizeof(int))) == cudaSuccess &&
        (e = cudaMemset(kv->gave_up, 0, sizeof(int))) == cudaSuccess &&
        (e = each_kernel([](auto kern, size_t smem) {
           return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
         })) == cudaSuccess)
      e = cudaDeviceSynchronize();
  }
  if (rc || e != cudaSuccess) {
    kv->mem.release();
    delete kv;
    return rc ? rc : set_error(GRID_E_CUDA, std::string("grid_kv_create: ") + cudaGetErrorString(e));
  }
  *out = kv;
  return GRID_OK;
}

extern "C" void grid_kv_free(grid_kv* kv) {
  if (!kv) return;
  kv->mem.release();
  delete kv;
}

extern "C" int grid_kv_attend(const grid_kv* kv, const grid_kv_chunk* chunk, const grid_kv_query* query,
                              int32_t* d_status, void* stream) {
  AttendArgs a = {};
  if (!kv || !query || !d_status || !make_chunk(kv, chunk, a.c) ||
      (chunk->n_tokens && (!heads_ok(&query->q) || !heads_ok(&query->out))) || !std::isfinite(query->scale) ||
      !(query->scale > 0.f) || (uintptr_t)query->d_lse % 4)
    return set_error(GRID_E_INVALID_ARG, "grid_kv_attend: bad arguments");
  if (chunk->B > 65535) return set_error(GRID_E_TOO_LARGE, "grid_kv_attend: more than 65535 rows");
  const grid_kv_pages& p = kv->p;
  // (more than two billion tiles of 256 query rows by 128 keys would take minutes)
  const double units = (double)chunk->n_tokens * (p.n_heads / p.n_kv_heads) / 256 + chunk->B;
  if ((double)chunk->n_tokens * (p.n_heads / p.n_kv_heads) > INT32_MAX - 256 ||
      units * p.n_kv_heads * (((double)chunk->max_pages * p.page_size) / kTile + 1 + kUnitCost) > kMostCost)
    return set_error(GRID_E_TOO_LARGE, "grid_kv_attend: too many query rows or key tiles in one call");
  a.q = query->q.d, a.out = query->out.d, a.lse = query->d_lse;
  a.qs[0] = query->q.token_stride, a.qs[1] = query->q.head_stride;
  a.os[0] = query->out.token_stride, a.os[1] = query->out.head_stride;
  a.H = p.n_heads, a.Hk = p.n_kv_heads, a.group = a.H / a.Hk, a.scale = query->scale, a.status = d_status;
  a.sectors = (uintptr_t)a.out % 32 == 0 && a.os[0] % 16 == 0 && a.os[1] % 16 == 0;
  a.parts = reinterpret_cast<float4*>(kv->parts), a.part_ml = kv->part_ml, a.joined = kv->joined, a.gave_up = kv->gave_up;
  auto go = [&](auto kern, size_t smem) {
    return launch_pdl(kern, dim3(kv->sms), dim3(kThreads), smem, (cudaStream_t)stream, a, kv->k_map, kv->v_map);
  };
  if (p.dtype == GRID_DTYPE_BF16)
    GRID_CUDA(p.head_dim == 64 ? go(k_attend<__nv_bfloat16, 64>, smem_bytes<64>())
                               : go(k_attend<__nv_bfloat16, 128>, smem_bytes<128>()));
  else
    GRID_CUDA(p.head_dim == 64 ? go(k_attend<__half, 64>, smem_bytes<64>()) : go(k_attend<__half, 128>, smem_bytes<128>()));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}
