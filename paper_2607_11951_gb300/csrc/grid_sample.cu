// Sampling from a masked distribution cut by top-k, top-p and min-p, from given
// random numbers (grid_sample).
//
// With m the row's largest admitted logit and c = log2(e) / T, an id's weight is
// w = 2^((l - m) c), its probability w / Z with Z the sum over the admitted ids.
// Ids are ordered by one 54-bit number, the logit's bits in the order of integers
// and then the id's complement, so that what top-k and top-p keep is "order >=
// X".
//
// A cluster of blocks per row holds the row's admitted logits in its shared
// memory: each logit is read from memory once, noise only where an id is kept.
// Each block learns what the others found and goes on for itself, so that a
// step costs one barrier of the cluster.  X is found in up to three steps:
//   - Ids that cannot be at the cut are left out: below the k-th largest of the
//     threads' largest logits; or (top-p alone) of less than (1 - top_p) Z / ids,
//     which together have less than 1 - top_p.
//   - The others go into 1,024 bins of equal width in m - l, with the number and
//     the weight of each, and the bin is found in which the k-th id, or top_p of
//     the weight, is reached.
//   - That bin's ids are sorted, and X is one of them.  A bin of more than a list
//     holds, as equal logits make it, is cut into 512 parts of its range of order
//     instead, and again: nine bits less each time, six times at most.
// For a small top-k, or where few ids are admitted, all that is left after the
// first step is sorted, and block 0 draws from the list.  min-p needs no X: its
// bound on (m - l) c is asked of every id.
//
// A block whose mask admits few ids takes those alone, one after the other (one
// such row over 151,936 ids: 8.2 us instead of 11.2); rows without masks have
// kernels of their own, which look at no bits.
//
// Sums of weights are integers, so that the order of the atomic additions does not
// matter: in a bin in steps of 2^-16 or less of its weights (what fits 32 bits if
// all of a block's ids are in it), elsewhere of 2^-40 of the largest.
//
// The end of a nucleus that is found by bins may be off by what rounding a share
// to 1 / scale gives, 2.3e-6 of the weight before it at 151,936 ids and 6e-6 at
// 393,216 (the same for all ids of one logit), and by the exponents' roundings.
// top-k's count is exact, whatever top-p asks for beside it.
//
// Bound by steps that follow one another (a row over 151,936 ids takes 9 to 21 us
// alone, of which the loads are 3 and each barrier of the cluster 0.7) and, where
// many rows share the SMs, by the instructions for an id and the additions to bins.
// In a graph: 32 fp32 rows over 151,936 ids (20 MB) with settings of all kinds take
// 28 us, 256 bf16 rows (83 MB) 72 to 77, one row over 512 ids 3.0 (no cut) to 6.6
// (top-p).  Without cuts 32 rows take 11.6, most of it for the noise (39 MB).
#include <atomic>
#include <cfloat>
#include <climits>
#include <cmath>

#include <cuda_bf16.h>

#include "grid_model.cuh"

namespace grid {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxBlocks = 8;             // of a row: the largest cluster that every device takes
constexpr int kBins = 1024, kPer = kBins / kThreads;  // a thread sums up kPer neighbours
constexpr int kParts = 512, kPartBits = 9;            // of a range of order
constexpr int kList = 512;                // ids that are sorted at once
constexpr int kCounted = 128;             // ids that are sorted by counting (one row of 128: 5.8 us, 6.6 by the network; of 250 7.3, 7.2)
constexpr unsigned kFew = 128;            // admitted ids that are sorted in any case (one row of 512, top_k 50: 5.0 us, sorted 7.5)
constexpr int kDirect = 256;              // a top_k up to here is looked for without bins (250, 32 rows over 151,936 ids: 18.0 us, with bins 22.6)
constexpr int kSparse = 2048;             // admitted ids of a block that are taken one by one, if an eighth of all at most
constexpr int kIdBits = 22;
constexpr int kMaxIds = 393216;           // 48 Ki fp32 logits for each of eight blocks
constexpr float kFirstRange = 40.f;       // exponents below m that bins reach
constexpr float kUnit = 1099511627776.f;  // 2^40
constexpr float kWhole = 8388608.f;       // 2^23: floats from here on are whole numbers
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
using u64 = unsigned long long;

struct SampleArgs {
  grid_sample_step s;
  int each;   // ids of a block (a multiple of 32)
  int sorted; // rows that take long go first
};

// What a row asks for.
struct Ask {
  float temp, top_p, min_p;
  int top_k;
  bool greedy, first;  // first: only the first id is kept
};
__device__ __forceinline__ Ask ask_of(const grid_sample_step& s, int b) {
  Ask a;
  a.temp = s.d_temperature ? s.d_temperature[b] : 1.f;
  a.top_k = s.d_top_k ? s.d_top_k[b] : 0;
  a.top_p = s.d_top_p ? s.d_top_p[b] : 1.f, a.min_p = s.d_min_p ? s.d_min_p[b] : 0.f;
  a.greedy = !(a.temp > 0.f);
  a.first = a.greedy || a.top_k == 1 || a.top_p <= 0.f || a.min_p > 1.f;
  return a;
}

struct Pick {   // of a draw: the best score, its id and logit; the first id of the largest logit
  float score, logit;
  int id, first;
};
struct Found {  // the bin that a search ends in, and what lies in the bins before it
  int bin;
  unsigned count;
  u64 weight;
};

struct Shared {
  union {
    float tops[kMaxBlocks * kThreads];     // of all threads of the row: their largest logits
    struct {
      unsigned n[kBins], w[kBins];         // ids and weights
    } bins;
    struct {
      unsigned n[kParts], lo[kParts], hi[kParts];  // the weights in 64 bits
    } parts;
    u64 other[kList];                      // of a list that is sorted
  };
  u64 list[2][kList];                      // of one gathering and the next: a block's ids in a part of its own
  // what every block of the row writes here
  float top[kMaxBlocks], low[kMaxBlocks];  // its largest admitted logit, the smallest of its threads' largest (negative)
  unsigned ids[kMaxBlocks];                // admitted
  float z[kMaxBlocks];                     // sum of weights
  unsigned in[2][kMaxBlocks];              // ids in the range that is gathered
  u64 most[kMaxBlocks], least[kMaxBlocks]; // the first and the last (~) of them
  Pick pick[kMaxBlocks];                   // (block 0)
  // of the block alone
  Found found;
  u64 target, kept;
  unsigned staged, at;
  int row;
  u64 sums[kWarps], sums2[kWarps];
  float3 warps[kWarps];
  float zw[kWarps];
  Pick picks[kWarps];
};
constexpr int kSharedRoom = (sizeof(Shared) + 127) & ~127;

__device__ __forceinline__ int cluster_rank() {
  int r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Block r's copy of something in shared memory.
__device__ __forceinline__ uint32_t there(const void* p, int r) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(r));
  return at;
}
__device__ __forceinline__ uint4 get4(const unsigned* x, int r) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(there(x, r)));
  return v;
}
__device__ __forceinline__ void put(unsigned& x, unsigned v, int r) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there(&x, r)), "r"(v) : "memory");
}
__device__ __forceinline__ void put(int& x, int v, int r) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there(&x, r)), "r"(v) : "memory");
}
__device__ __forceinline__ void put(float& x, float v, int r) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there(&x, r)), "f"(v) : "memory");
}
__device__ __forceinline__ void put(u64& x, u64 v, int r) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there(&x, r)), "l"(v) : "memory");
}

__device__ __forceinline__ u64 max_warp(u64 x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = max(x, __shfl_xor_sync(~0u, x, o));
  return x;
}
__device__ __forceinline__ float max_warp(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, o));
  return x;
}
__device__ __forceinline__ float sum_warp(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  return x;
}
__device__ __forceinline__ void better(Pick& x, const Pick& y) {
  if (y.score < x.score || (y.score == x.score && y.id < x.id)) x.score = y.score, x.logit = y.logit, x.id = y.id;
  x.first = min(x.first, y.first);
}
__device__ __forceinline__ Pick best_warp(Pick x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const Pick y = {__shfl_xor_sync(~0u, x.score, o), __shfl_xor_sync(~0u, x.logit, o), __shfl_xor_sync(~0u, x.id, o),
                    __shfl_xor_sync(~0u, x.first, o)};
    better(x, y);
  }
  return x;
}
// The sum over the block's threads up to this one, and over all of them.
template <typename N>
__device__ __forceinline__ N up_to(N x, u64* sums, N& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const N y = __shfl_up_sync(~0u, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();  // (`sums` may still be read from the last time)
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const N y = (N)sums[w];
    if (w < warp) x += y;
    all += y;
  }
  return x;
}

// Sixteen bytes of logits: NaN as -inf, +inf as the largest finite value of the type, and -inf where the bit is not set; the
// largest of them; the values in pairs.
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }  // bf16
__device__ __forceinline__ float kept_as(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX); }
__device__ __forceinline__ uint16_t kept_as(uint16_t x) { return (x & 0x7FFF) > 0x7F80 ? 0xFF80 : x == 0x7F80 ? 0x7F7F : x; }
template <typename T>
struct Line;
template <>
struct Line<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float none() { return -INFINITY; }
  static __device__ __forceinline__ uint4 admit(const uint4& r, unsigned bits) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    uint32_t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = bits >> e & 1u ? __float_as_uint(kept_as(__uint_as_float(w[e]))) : 0xFF800000u;
    return make_uint4(y[0], y[1], y[2], y[3]);
  }
  static __device__ __forceinline__ float top(const uint4& r) {
    return fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w)));
  }
  static __device__ __forceinline__ Two pair(const uint4& r, int e) {
    return e ? Two{__uint_as_float(r.z), __uint_as_float(r.w)} : Two{__uint_as_float(r.x), __uint_as_float(r.y)};
  }
};
template <>
struct Line<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ uint16_t none() { return 0xFF80; }
  // Four bytes, each the top bit of one of x's eight times.
  template <int kOf>
  static __device__ __forceinline__ uint32_t signs(uint32_t x) {
    uint32_t y;
    asm("prmt.b32 %0, %1, 0, %2;" : "=r"(y) : "r"(x), "n"(kOf));
    return y;
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 v = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  static __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 v = __hmin2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  static __device__ __forceinline__ uint4 admit(const uint4& r, unsigned bits) {
    // (four bits to the tops of four bytes: bit i goes to i + 7, i + 14, i + 21 and i + 28, which never meet; then each top
    // bit twice as a byte of its own, two bytes for a value)
    const uint32_t lo = (bits & 15u) * 0x10204080u, hi = (bits >> 4) * 0x10204080u;
    const uint32_t in[4] = {signs<0x9988>(lo), signs<0xBBAA>(lo), signs<0x9988>(hi), signs<0xBBAA>(hi)};
    uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (min2(max2(w[e], 0xFF80FF80u), 0x7F7F7F7Fu) & in[e]) | (0xFF80FF80u & ~in[e]);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float top(const uint4& r) {
    const uint32_t x = max2(max2(r.x, r.y), max2(r.z, r.w));
    return fmaxf(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
  }
  static __device__ __forceinline__ Two pair(const uint4& r, int e) {
    const uint32_t w = e == 0 ? r.x : e == 1 ? r.y : e == 2 ? r.z : r.w;
    return Two{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)};
  }
};
// A load where `in` holds, without a branch: as branches, the loads of a loop wait for one another.
__device__ __forceinline__ void load_if(float& x, const float* p, bool in) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\n@p ld.global.nc.f32 %0, [%1];\n}" : "+f"(x) : "l"(p), "r"((int)in));
}
__device__ __forceinline__ void load_if(uint4& x, const void* p, bool in) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %5, 0;\n@p ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
               : "+r"(x.x), "+r"(x.y), "+r"(x.z), "+r"(x.w)
               : "l"(p), "r"((int)in));
}

// The logit's bits in the order of integers, then the id's complement; and back.
__device__ __forceinline__ u64 order_of(float x, int id) {
  const unsigned b = __float_as_uint(x + 0.f);  // (-0 is 0)
  return (u64)(b ^ ((unsigned)((int)b >> 31) | 0x80000000u)) << kIdBits | (unsigned)((1 << kIdBits) - 1 - id);
}
__device__ __forceinline__ float logit_of(u64 o) {
  const unsigned k = (unsigned)(o >> kIdBits);
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

__device__ __forceinline__ int id_of(u64 o) { return (1 << kIdBits) - 1 - (int)(o & ((1u << kIdBits) - 1u)); }

// A row's weights and bins.
struct Row {
  float c2;     // 2 log2(e) / T
  float m, by;  // the largest logit; bins per half of m - l
  float width;  // exponents of a bin
  // half of m - l: of the halves, since the difference of two logits may be past the type
  __device__ __forceinline__ float below(float x) const { return fmaf(0.5f, m, -0.5f * x); }
  __device__ __forceinline__ float weight(float x) const { return exp2_fast(-below(x) * c2); }
  // Where it lies among the bins, and the nearest one: a whole number in the low bits of a float of 2^23 and more (conversions
  // run at an eighth of an addition's rate).
  __device__ __forceinline__ float place(float x) const { return fminf(below(x) * by, (float)(kBins - 1)); }
  static __device__ __forceinline__ int low(float whole) { return __float_as_int(whole) & 0x7FFFFF; }
  __device__ __forceinline__ int bin(float x) const { return low(place(x) + kWhole); }
  __device__ __forceinline__ void reach(float range) {  // bins of halves of m - l up to `range`
    range = fminf(range, fminf(kFirstRange / c2, FLT_MAX));
    by = range > 0.f ? fminf(kBins / range, FLT_MAX) : 0.f;
    width = c2 / by;
    if (!(by > 0.f)) width = 0.f;  // (all of one logit)
  }
  // The weight in a bin's middle.
  __device__ __forceinline__ float middle(int bin) const { return exp2_fast(-(float)bin * width); }
  // Nothing below this has a half of m - l of up to h: the roundings of both, 2^-23 of h or of a logit, are allowed for.
  __device__ __forceinline__ float least(float h) const { return m - 2.f * h - 1e-6f * (h + fabsf(m)); }
  // Nothing above this has one of h or more.
  __device__ __forceinline__ float most(float h) const { return m - 2.f * h + 1e-6f * (h + fabsf(m)); }
};
__device__ __forceinline__ u64 units(float w) { return __float2ull_rn(w * kUnit); }

template <typename T, int blocks, bool kMasked>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 2) k_sample(const SampleArgs a) {
  using L = Line<T>;
  constexpr int N = L::N;
  extern __shared__ __align__(128) uint8_t raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  uint4* const lines = reinterpret_cast<uint4*>(raw + kSharedRoom);
  const grid_sample_step& s = a.s;
  const int rank = cluster_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lo = min(s.V, rank * a.each), n = min(s.V, lo + a.each) - lo;
  auto sync = [&]() {  // of the row's blocks
    __syncwarp();
    if (blocks > 1)
      asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else
      __syncthreads();
  };
  if (blocks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  if (tid == 0) sh.at = 0, sh.found = Found{0, 0u, 0ull};  // (inside the list and the bins, whatever is found)
  pdl_wait();
  int b = blockIdx.x / blocks;
  if (a.sorted) {  // the b-th in the order: rows cut by top-p or a large top-k, uncut ones, those of one id
    const int per = (s.B + kThreads - 1) / kThreads;
    u64 mine = 0;  // rows of each kind, 16 bits apart
    auto kind = [&](int i) {
      const Ask x = ask_of(s, i);
      return x.first ? 32 : x.top_p < 1.f || x.top_k > kDirect ? 0 : 16;
    };
    for (int i = tid * per; i < min(s.B, (tid + 1) * per); ++i) mine += 1ull << kind(i);
    u64 all, at = up_to(mine, sh.sums, all) - mine;
    const int n0 = (int)(all & 0xFFFF), n1 = (int)(all >> 16 & 0xFFFF);
    const int of = b < n0 ? 0 : b < n0 + n1 ? 16 : 32, nth = b - (of == 0 ? 0 : of == 16 ? n0 : n0 + n1);
    if ((int)(at >> of & 0xFFFF) <= nth && nth < (int)((at + mine) >> of & 0xFFFF))
      for (int i = tid * per, k = (int)(at >> of & 0xFFFF); i < min(s.B, (tid + 1) * per); ++i)
        if (kind(i) == of && k++ == nth) sh.row = i;
    __syncthreads();
    b = sh.row;
  }
  const Ask ask = ask_of(s, b);
  const int top_k = ask.top_k;
  const float temp = ask.temp, top_p = ask.top_p, min_p = ask.min_p;
  const bool greedy = ask.greedy, first = ask.first;
  Row row;
  row.c2 = fminf((greedy ? 1.f : 1.f / temp) * (2.f * kLog2e), 1e37f);  // (so that 1,024 bins of 40 exponents have a width)

  // ---- the block's logits in lines of 16 bytes as they lie in memory: line v holds the block's ids v N - pad .. + N - 1
  // (where few of them are admitted, `taken`: those alone, one after the other, and behind them their places in the block)
  int pad = 0, count_v = 0, taken = -1;
  float top = -INFINITY;  // the thread's largest logit, and the first of its lines that has it
  int top_v = 0;
  unsigned ids = 0;
  auto places = [&]() { return reinterpret_cast<uint16_t*>(lines + (taken * (int)sizeof(T) + 15) / 16); };
  auto id_at = [&](int i) { return lo + (taken >= 0 ? (int)places()[i] : i); };
  {
    const T* l = static_cast<const T*>(s.d_logits) + b * s.logit_stride + lo;
    const uint32_t* mask = kMasked ? s.d_mask + b * s.mask_stride + (lo >> 5) : nullptr;
    pad = (int)((uintptr_t)l & 15) / (int)sizeof(T);
    count_v = n > 0 ? (pad + n + N - 1) / N : 0;
    const int inner = n - N;  // a whole line begins at an id of 0 .. inner
    // The mask's words first, so that no logit waits for its bit (the lists are not in use yet); then all whole lines that
    // hold an admitted id at once, each by the thread that takes it on.
    uint32_t* const words = reinterpret_cast<uint32_t*>(sh.list);
    static_assert(kMaxIds / kMaxBlocks / 32 < 4 * kList);
    if (mask) {
      const int whole = (n + 31) / 32;
      for (int w = tid; w <= whole; w += kThreads)
        words[w] = w < whole ? mask[w] & (32 * w + 32 > n ? (1u << (n - 32 * w)) - 1u : ~0u) : 0u;
      __syncthreads();
      if (blocks > 1) {  // (a block alone is soon through: one row over 512 ids would take 0.5 us more)
        const int per = (whole + kThreads - 1) / kThreads, w0 = min(whole, tid * per), w1 = min(whole, w0 + per);
        unsigned mine = 0, all;
        for (int w = w0; w < w1; ++w) mine += __popc(words[w]);
        unsigned at = up_to(mine, sh.sums, all) - mine;
        if (all <= kSparse && all * 8 <= (unsigned)n) {
          taken = (int)all, pad = 0, count_v = (taken + N - 1) / N;
          for (int w = w0; w < w1; ++w)
            for (unsigned bits = words[w]; bits; bits &= bits - 1) places()[at++] = (uint16_t)(32 * w + __ffs(bits) - 1);
          __syncthreads();
          for (int i = tid; i < count_v * N; i += kThreads) {
            T x = L::none();
            if (i < taken) x = kept_as(l[places()[i]]), ++ids;
            if (value(x) > top) top = value(x), top_v = i / N;
            reinterpret_cast<T*>(lines)[i] = x;
          }
        }
      }
    }
    if (taken < 0) {
      auto bits_of = [&](int v) {
        const int i = v * N - pad;
        if (i < 0 || i > inner) return 0u;
        return mask ? __funnelshift_r(words[i >> 5], words[(i >> 5) + 1], i & 31) & ((1u << N) - 1u) : (1u << N) - 1u;
      };
#pragma unroll 4
      for (int v = tid; v < count_v; v += kThreads)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\n@p cp.async.cg.shared.global [%0], [%1], 16;\n}" ::"r"(
                         (uint32_t)__cvta_generic_to_shared(lines + v)),
                     "l"(l + (v * N - pad)), "r"(bits_of(v))
                     : "memory");
      asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 2
      for (int v = tid; v < count_v; v += kThreads) {
        const unsigned bits = bits_of(v);
        const uint4 x = L::admit(lines[v], bits);
        lines[v] = x;
        const float t = L::top(x);
        if (t > top) top = t, top_v = v;
        ids += __popc(bits);
      }
      // lines that are not whole: the first and the last, an id to a thread
      __syncthreads();
      if (tid < 2 * N && count_v > 0 && (tid < N || count_v > 1)) {
        const int v = tid < N ? 0 : count_v - 1, i = v * N + tid % N - pad;
        if (v * N - pad < 0 || v * N - pad > inner) {
          T x = L::none();
          if (i >= 0 && i < n && (!mask || words[i >> 5] >> (i & 31) & 1u)) {
            x = kept_as(l[i]);
            ++ids;
          }
          reinterpret_cast<T*>(lines + v)[tid % N] = x;
          if (value(x) > top || (v == 0 && value(x) == top)) top = value(x), top_v = v;
        }
      }
    }
  }
  // f(x, i) for the block's ids i whose logit x is admitted and at least `from`
  auto each = [&](float from, auto f) {
    from = fmaxf(from, -FLT_MAX);
    for (int v = tid; v < count_v; v += kThreads) {
      const uint4 r = lines[v];
      if (!(L::top(r) >= from)) continue;
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const Two x = L::pair(r, e / 2);
        if (x.x >= from) f(x.x, v * N + e - pad);
        if (x.y >= from) f(x.y, v * N + e + 1 - pad);
      }
    }
  };

  // ---- the block's largest logit and the sum of its weights, relative to that; then, over the row's blocks: the largest
  // logit, the sum, all threads' largest, the smallest of those, how many ids are admitted
  const bool wants_k = !first && top_k > 0;
  unsigned* const top_bins = reinterpret_cast<unsigned*>(sh.list[0]);  // (the first list is the other one)
  static_assert(sizeof(sh.list[0]) >= kBins * sizeof(unsigned));
  float all_z = 0.f;
  {
    const float t = max_warp(top), u = max_warp(top > -INFINITY ? -top : -INFINITY);
    const unsigned c = __reduce_add_sync(~0u, ids);
    if (lane == 0) sh.warps[warp] = make_float3(t, u, __uint_as_float(c));
    __syncthreads();
    float m = -INFINITY, z = 0.f;
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sh.warps[w].x);
    if (!(m > -INFINITY)) {
    } else if (row.c2 > 0.f) {
      Two sum = {0.f, 0.f};
#pragma unroll 2
      for (int v = tid; v < count_v; v += kThreads) {
        const uint4 r = lines[v];
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          const Two t = mul2(fma2(L::pair(r, e), 0.5f, -0.5f * m), Two{row.c2, row.c2});
          sum = add2(sum, Two{exp2_fast(t.x), exp2_fast(t.y)});
        }
      }
      z = sum.x + sum.y;
    } else {  // (T is infinite: all finite logits weigh the same)
      each(-INFINITY, [&](float, int) { z += 1.f; });
    }
    z = sum_warp(z);
    if (lane == 0) sh.zw[warp] = z;
    for (int i = tid; i < kBins; i += kThreads) top_bins[i] = 0;
    __syncthreads();
    if (blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // (the others are there)
    if (wants_k)
      for (int r = 0; r < blocks; ++r) put(sh.tops[rank * kThreads + tid], top, r);
    if (tid < blocks) {
      float y = -INFINITY;
      unsigned all = 0;
      z = 0.f;
      for (int w = 0; w < kWarps; ++w) y = fmaxf(y, sh.warps[w].y), all += __float_as_uint(sh.warps[w].z), z += sh.zw[w];
      put(sh.top[rank], m, tid);
      put(sh.low[rank], y, tid);
      put(sh.ids[rank], all, tid);
      put(sh.z[rank], z, tid);
    }
    sync();
  }
  ids = 0;
  row.m = -INFINITY;
  for (int r = 0; r < blocks; ++r) row.m = fmaxf(row.m, sh.top[r]), ids += sh.ids[r];
  if (!(row.m > -INFINITY)) {  // (the same in every block)
    if (rank == 0 && tid == 0) {
      s.d_tokens[b] = -1;
      if (s.d_logprob) s.d_logprob[b] = 0.f;
      s.d_status[b] = GRID_ST_EMPTY_MASK;
    }
    return;
  }
  for (int r = 0; r < blocks; ++r)
    if (sh.top[r] > -INFINITY) all_z += sh.z[r] * row.weight(sh.top[r]);

  // (min-p by the exponent: the difference comes first, so that it holds at every temperature)
  const float t_most = min_p > 0.f ? -log2f(min_p) : INFINITY;
  auto write = [&](int token, float x) {
    s.d_tokens[b] = token;
    if (s.d_logprob) s.d_logprob[b] = fminf((-row.below(x) * row.c2 - log2f(all_z)) * kLn2, 0.f);
    s.d_status[b] = token == s.eos ? GRID_ST_COMPLETE : GRID_ST_OK;
  };

  // ---- the cut X: ids of order X and more are kept
  const bool by_k = wants_k && (unsigned)top_k < ids, by_p = !first && top_p < 1.f;
  u64 cut = 0;
  if (by_k || by_p) {
    const Found none = {0, 0u, 0ull};
    constexpr unsigned room = kList / blocks;  // of a block in a list
    int turn = 0;                          // which list
    // The list of all ids in a range, `in`, whose logits lie in from .. to; how many there are (more than kList: no list).
    auto gather = [&](float from, float to, auto in) {
      turn ^= 1;
      u64* list = sh.list[turn];
      if (tid == 0) sh.staged = 0;
      __syncthreads();
      from = fmaxf(from, -FLT_MAX);
      for (int v = tid; v < count_v; v += kThreads) {
        const uint4 r = lines[v];
        if (!(L::top(r) >= from)) continue;
        unsigned some = 0;
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const Two x = L::pair(r, e / 2);
          some |= (x.x >= from && x.x <= to ? 1u << e : 0u) | (x.y >= from && x.y <= to ? 2u << e : 0u);
        }
        for (; some; some &= some - 1) {
          const int e = __ffs(some) - 1;
          const float x = value(reinterpret_cast<const T*>(lines + v)[e]);
          const u64 o = order_of(x, id_at(v * N + e - pad));
          if (*(volatile unsigned*)&sh.staged > room || !in(x, o)) continue;  // (too many already: no need to look further)
          const unsigned at = atomicAdd(&sh.staged, 1u);
          if (at < room) list[rank * room + at] = o;
        }
      }
      __syncthreads();
      const unsigned mine = sh.staged;
      if (tid < blocks) put(sh.in[turn][rank], mine, tid);
      if (mine <= room)
        for (unsigned x = tid; x < mine * blocks; x += kThreads) {
          const unsigned r = x % blocks, at = rank * room + x / blocks;
          if (r != (unsigned)rank) put(list[at], list[at], r);
        }
      sync();
      unsigned all = 0, most = 0;
      for (int r = 0; r < blocks; ++r) all += sh.in[turn][r], most = max(most, sh.in[turn][r]);
      return most > room ? kList + 1u : all;
    };
    // The list in one piece and sorted.  Up to kCounted ids: an id's place is the number of those before it.  More: by a network
    // of comparisons, id i of 64 warp + 32 y + lane; partners 32 apart are in one thread, nearer ones in one warp, others meet in
    // shared memory, in two places by turns (a step costs one barrier; nobody looks at bins now).
    auto sort = [&](unsigned listed) {
      u64* list = sh.list[turn];
      auto listed_at = [&](unsigned i) {
        unsigned r = 0;
        const bool in = i < listed;
        while (r + 1 < (unsigned)blocks && i >= sh.in[turn][r]) i -= sh.in[turn][r++];
        return in ? list[r * room + i] : 0ull;
      };
      if (listed <= kCounted) {
        const u64 mine = tid < kCounted ? listed_at(tid) : 0;
        __syncthreads();
        if (tid < kCounted) list[tid] = mine;
        __syncthreads();
        unsigned place = 0;
        if (warp * 32 < listed)
#pragma unroll 4
          for (unsigned i = 0; i < listed; i += 2) {  // (zeros past the last)
            const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(list + i);
            place += (o.x > mine) + (o.y > mine);
          }
        __syncthreads();
        if (tid < listed) list[place] = mine;
        __syncthreads();
        return;
      }
      unsigned size = 64;
      while (size < listed) size *= 2;
      const unsigned i0 = 64 * warp + lane;
      const bool in = 64 * warp < size;
      u64 x[2] = {};
      if (in) x[0] = listed_at(i0), x[1] = listed_at(i0 + 32);
      bool apart = false;  // where the last values were put
      for (unsigned k = 2; k <= size; k *= 2) {
        for (unsigned j = k / 2; j >= 64; j /= 2) {
          apart = !apart;
          u64* at = apart ? sh.other : list;
          if (in) at[i0] = x[0], at[i0 + 32] = x[1];
          __syncthreads();
          if (in) {
            const bool most = ((i0 & k) == 0) == ((i0 & j) == 0);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const u64 o = at[(i0 ^ j) + 32 * y];
              x[y] = (o > x[y]) == most ? o : x[y];
            }
          }
        }
        if (!in) continue;
        if (k >= 64 && (x[0] > x[1]) != ((i0 & k) == 0)) {
          const u64 o = x[0];
          x[0] = x[1], x[1] = o;
        }
        for (unsigned j = min(k / 2, 16u); j; j /= 2)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const bool most = (((i0 + 32 * y) & k) == 0) == ((lane & j) == 0);
            const u64 o = __shfl_xor_sync(~0u, x[y], j);
            x[y] = (o > x[y]) == most ? o : x[y];
          }
      }
      if (!apart) __syncthreads();
      if (in) list[i0] = x[0], list[i0 + 32] = x[1];
      __syncthreads();
    };
    // The last id of the sorted list that a target needs, if so much comes before the list (the list's last where roundings
    // leave the target a little out of reach): its place, and the weight up to it.
    auto last_of = [&](unsigned listed, bool weights, u64 target, const Found& f) {
      u64 weight = f.weight;
      for (unsigned i0 = 0; i0 < listed; i0 += kThreads) {
        const unsigned i = i0 + tid;
        const bool some = i < listed;
        const u64 w = some && by_p ? units(row.weight(logit_of(sh.list[turn][i]))) : 0;
        u64 all;
        const u64 upto = up_to(w, sh.sums, all);
        const u64 was = weights ? weight + upto - w : f.count + (u64)i, now = weights ? weight + upto : f.count + (u64)i + 1;
        if (some && was < target && (now >= target || i + 1 == listed)) sh.at = i, sh.kept = weight + upto;
        weight += all;
      }
      __syncthreads();
    };
    auto target_of = [&](u64 sum) {
      __syncthreads();
      if (tid == 0) sh.target = max((u64)ceil((double)top_p * (double)sum), 1ull);
      __syncthreads();
      return sh.target;
    };
    // The cut from the list: by count, by weight (a target of 0: its share of what is listed, or kept by count), or by both.
    auto cut_from = [&](unsigned listed, bool k, bool p, u64 target, const Found& f) {
      sort(listed);
      if (k || !target) {
        last_of(listed, false, k ? top_k : f.count + listed, f);
        listed = sh.at + 1;
      }
      if (p) last_of(listed, true, target ? target : target_of(sh.kept), f);
      return sh.list[turn][sh.at];
    };
    // Of the bins kPer tid .. + kPer - 1 of all blocks: the ids and the weight up to and with each.
    unsigned upto_n[kPer];
    u64 upto_w[kPer];
    // bf16 logits from `from` on that are positive and of no more values than there are bins have a bin for each value, the
    // largest's first: only their numbers are counted (256 rows with top-p were 120 us instead of 125)
    bool by_value = false;
    const int top_value = __float_as_int(row.m) >> 16;
    auto value_of = [&](int bin) { return __int_as_float((top_value - bin) << 16); };
    auto sum_up = [&](const unsigned* n, const unsigned* w, const unsigned* high, float scale) {
      u64 low[kPer] = {}, up[kPer] = {};
      unsigned cn[kPer] = {};
      auto add = [&](const unsigned* of, auto& sums) {
#pragma unroll
        for (int r0 = 0; r0 < blocks; r0 += 4) {  // (four blocks' at once)
          constexpr int kAt = blocks < 4 ? blocks : 4;
          uint4 x[kAt];
#pragma unroll
          for (int r = 0; r < kAt; ++r) x[r] = get4(of + kPer * tid, r0 + r);
#pragma unroll
          for (int r = 0; r < kAt; ++r) sums[0] += x[r].x, sums[1] += x[r].y, sums[2] += x[r].z, sums[3] += x[r].w;
        }
      };
      if (!high || kPer * tid < kParts) {
        if (n) add(n, cn);
        if (w) add(w, low);
        if (high) add(high, up);
      }
      unsigned sum_n = 0, all_n;
      u64 sum_w = 0, all_w;
#pragma unroll
      for (int y = 0; y < kPer; ++y) {
        u64 x = low[y] + (up[y] << 32);
        if (!high && by_value)
          x = cn[y] ? cn[y] * units(row.weight(value_of(kPer * tid + y))) : 0;
        else if (!high)
          x = __float2ull_rn((float)x * (row.middle(kPer * tid + y) * scale));
        sum_n += cn[y], sum_w += x;
        upto_n[y] = sum_n, upto_w[y] = sum_w;
      }
      const unsigned before_n = up_to(sum_n, sh.sums, all_n) - sum_n;
      const u64 before_w = up_to(sum_w, sh.sums2, all_w) - sum_w;
#pragma unroll
      for (int y = 0; y < kPer; ++y) upto_n[y] += before_n, upto_w[y] += before_w;
      return Found{0, all_n, all_w};
    };
    // The bin in which, after `before`, the target is reached (it is reached in one).
    auto search = [&](bool weights, u64 target, const Found& f) {
      __syncthreads();
      unsigned was_n = __shfl_up_sync(~0u, upto_n[kPer - 1], 1);
      u64 was_w = __shfl_up_sync(~0u, upto_w[kPer - 1], 1);
      if (lane == 31) sh.sums[warp] = upto_n[kPer - 1], sh.sums2[warp] = upto_w[kPer - 1];
      __syncthreads();
      if (lane == 0) was_n = warp ? (unsigned)sh.sums[warp - 1] : 0u, was_w = warp ? sh.sums2[warp - 1] : 0ull;
#pragma unroll
      for (int y = 0; y < kPer; ++y) {
        const u64 was = weights ? f.weight + was_w : f.count + (u64)was_n;
        const u64 now = weights ? f.weight + upto_w[y] : f.count + (u64)upto_n[y];
        if (was < target && now >= target) sh.found = Found{kPer * tid + y, f.count + was_n, f.weight + was_w};
        was_n = upto_n[y], was_w = upto_w[y];
      }
      __syncthreads();
      return sh.found;
    };
    bool ready = false;  // the sums are of the bins
    // X of a target among the bins, and the weight up to it.
    auto find = [&](float from, bool weights, u64 target, u64& kept) {
      Found f = search(weights, target, none);
      const int bin = f.bin;
      // (of equal logits or logits that are nearly so, there may be too many in a bin)
      float to = INFINITY;
      auto in_bin = [&](float x) { return by_value ? x == value_of(bin) : row.bin(x) == bin; };
      if (by_value) {
        from = to = value_of(bin);
      } else if (row.by > 0.f) {
        // (bins are rounded to the nearest whole number)
        if (bin < kBins - 1) from = fmaxf(from, row.least((bin + 0.5f) / row.by));
        if (bin > 0) to = row.most((bin - 0.5f) / row.by);
      }
      unsigned listed = gather(from, to, [&](float x, u64) { return in_bin(x); });
      if (listed > kList) {
        u64 most = 0, least = 0;  // (least: as the largest complement)
        each(from, [&](float x, int i) {
          const u64 o = order_of(x, id_at(i));
          if (in_bin(x)) most = max(most, o), least = max(least, ~o);
        });
        most = max_warp(most), least = max_warp(least);
        __syncthreads();
        if (lane == 0) sh.sums[warp] = most, sh.sums2[warp] = least;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) most = max(most, sh.sums[w]), least = max(least, sh.sums2[w]);
        if (tid < blocks) put(sh.most[rank], most, tid), put(sh.least[rank], least, tid);
        sync();
        for (int r = 0; r < blocks; ++r) most = max(most, sh.most[r]), least = max(least, sh.least[r]);
        least = ~least;
        ready = false;
        while (listed > kList) {
          const int shift = max(0, 64 - __clzll((long long)(most - least)) - kPartBits);
          for (int i = tid; i < kParts; i += kThreads) sh.parts.n[i] = sh.parts.lo[i] = sh.parts.hi[i] = 0;
          __syncthreads();
          each(from, [&](float x, int i) {
            const u64 o = order_of(x, id_at(i));
            if (o < least || o > most) return;
            const int part = (int)((most - o) >> shift);
            atomicAdd(&sh.parts.n[part], 1u);
            if (!by_p) return;
            const u64 w = units(row.weight(x));
            const unsigned l = (unsigned)w, was = l ? atomicAdd(&sh.parts.lo[part], l) : 0u;
            const unsigned h = (unsigned)(w >> 32) + (was + l < was);
            if (h) atomicAdd(&sh.parts.hi[part], h);
          });
          sync();
          const Found all = sum_up(sh.parts.n, sh.parts.lo, sh.parts.hi, 0.f);
          // (the bins' weights are rounded otherwise: what they promise may be a little out of reach)
          // (of ids that all weigh less than half a unit any may be the last)
          const bool some = weights && all.weight;
          f = search(some, some ? min(target, f.weight + all.weight) : weights ? f.count + 1ull : target, f);
          most -= (u64)f.bin << shift;
          if (most - least >> shift) least = most - ((1ull << shift) - 1);
          const u64 z = most, a = least;
          listed = gather(logit_of(a), logit_of(z), [&](float, u64 o) { return o >= a && o <= z; });
        }
      }
      const u64 x = cut_from(listed, !weights, weights, target, f);
      kept = sh.kept;
      return x;
    };

    // Ids at or above `from` are looked at.
    float from = -INFINITY;
    u64 target = 0;  // of top-p alone
    const bool few = ids <= min(room, kFew);  // all of them are sorted
    if (few) {
    } else if (by_k) {
      // the bin that the k-th largest of the threads' largest lies in
      float low = -INFINITY;
      for (int r = 0; r < blocks; ++r) low = fmaxf(low, sh.low[r]);
      const float range = row.below(-low);
      row.by = range > 0.f ? fminf(kBins / range, FLT_MAX) : 0.f;
#pragma unroll
      for (int r = 0; r < blocks; ++r) {
        const float x = sh.tops[r * kThreads + tid];
        if (x > -INFINITY) atomicAdd(&top_bins[row.bin(x)], 1u);
      }
      __syncthreads();
      const uint4 x = reinterpret_cast<const uint4*>(top_bins)[tid];
      unsigned all;
      const unsigned upto = up_to(x.x + x.y + x.z + x.w, sh.sums, all);
      unsigned at = upto - (x.x + x.y + x.z + x.w);
      const unsigned one[kPer] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int y = 0; y < kPer; ++y) {
        if (at < (unsigned)top_k && at + one[y] >= (unsigned)top_k) sh.found.bin = kPer * tid + y;
        at += one[y];
      }
      __syncthreads();
      if (all >= (unsigned)top_k && row.by > 0.f && sh.found.bin < kBins - 1) from = row.least((sh.found.bin + 0.5f) / row.by);
    } else {
      if (row.c2 > 0.f) from = row.least(-log2f(0.99f * (1.f - top_p) * (all_z / ids)) / row.c2);
      target = max(__float2ull_ru(top_p * all_z * kUnit), 1ull);
      by_value = sizeof(T) == 2 && from > 0.f && top_value - (__float_as_int(from) >> 16) < kBins;
    }
    if (few || (by_k && top_k <= kDirect)) {
      const unsigned listed = gather(from, INFINITY, [](float, u64) { return true; });
      if (listed <= kList) {  // what is kept is in the list: block 0 draws from it
        if (rank) return;
        cut_from(listed, by_k, by_p, 0, none);
        Pick p = {INFINITY, row.m, INT_MAX, 0};
        for (unsigned i = tid; i <= sh.at; i += kThreads) {
          const u64 o = sh.list[turn][i];
          const float x = logit_of(o), t = row.below(x) * row.c2, e = s.d_noise[b * s.noise_stride + id_of(o)];
          const float score = e * exp2_fast(t);
          if (e >= FLT_MIN && t <= t_most) better(p, Pick{score, x, id_of(o), 0});
        }
        p = best_warp(p);
        if (lane == 0) sh.picks[warp] = p;
        __syncthreads();
        if (warp == 0) {
          p = best_warp(sh.picks[lane % kWarps]);
          const bool drawn = p.score < INFINITY;
          if (lane == 0) write(drawn ? p.id : id_of(sh.list[turn][0]), drawn ? p.logit : row.m);
        }
        return;
      }
    }
    row.reach(from > -INFINITY ? row.below(from) : INFINITY);
    // A weight is held as its share of the one in its bin's middle, 2^(f width) for an id f bins before it, f in -1/2 .. 1/2: a
    // square in f is within 2^-21 of it (width is 40 / 1,024 at most).  So many units make a share of one.
    const float scale = truncf(fminf(4.1e9f / a.each, 8e6f)), tilt = 0.6931471805599453f * row.width;
    auto share = [&](float f) {  // (as a whole number)
      return Row::low(fmaf(f, fmaf(f, 0.5f * tilt * tilt * scale, tilt * scale), scale + kWhole));
    };
    Found all;
    u64 kept = 0;
    for (int weights = !by_k; weights <= (int)by_p; ++weights) {  // by count, then by weight
      if (!ready) {
        for (int i = tid; i < kBins; i += kThreads) sh.bins.n[i] = sh.bins.w[i] = 0;
        __syncthreads();
        const float at_least = fmaxf(from, -FLT_MAX);
        constexpr int kLines = 8 / N;
        if (by_value) {
          const int least = (__float_as_int(from) + 0xFFFF) >> 16;  // (as whole numbers, negative logits are below)
          for (int v = tid; v < count_v; v += kThreads) {
            const uint4 r = lines[v];
            if (!(L::top(r) >= from)) continue;
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int x0 = (int16_t)w[y], x1 = (int)w[y] >> 16;
              if (x0 >= least) atomicAdd(&sh.bins.n[top_value - x0], 1u);
              if (x1 >= least) atomicAdd(&sh.bins.n[top_value - x1], 1u);
            }
          }
        } else if (by_k && from > -INFINITY) {  // few ids in many lines
          for (int v = tid; v < count_v; v += kThreads) {
            const uint4 r = lines[v];
            if (!(L::top(r) >= at_least)) continue;
            unsigned some = 0;
#pragma unroll
            for (int e = 0; e < N; e += 2) {
              const Two x = L::pair(r, e / 2);
              some |= (x.x >= at_least ? 1u << e : 0u) | (x.y >= at_least ? 2u << e : 0u);
            }
            for (; some; some &= some - 1) {
              const float x = value(reinterpret_cast<const T*>(lines + v)[__ffs(some) - 1]);
              const float at = row.place(x), in = at + kWhole;
              atomicAdd(&sh.bins.n[Row::low(in)], 1u);
              if (by_p) atomicAdd(&sh.bins.w[Row::low(in)], (unsigned)share(in - kWhole - at));
            }
          }
        } else
        for (int v0 = tid; v0 < count_v; v0 += kLines * kThreads) {  // eight ids at once: what one waits for, the others do too
          float x[8];
          int bin[8], w[8];
          bool any = false;
#pragma unroll
          for (int y = 0; y < 8; y += 2) {
            const int v = v0 + y / N * kThreads;
            const Two t = v < count_v ? L::pair(lines[v], y % N / 2) : Two{-INFINITY, -INFINITY};
            x[y] = t.x, x[y + 1] = t.y;
            any = any || fmaxf(t.x, t.y) >= at_least;
          }
          if (!any) continue;
#pragma unroll
          for (int y = 0; y < 8; y += 2) {
            Two at = mul2(fma2(Two{x[y], x[y + 1]}, -0.5f, 0.5f * row.m), Two{row.by, row.by});
            at = Two{fminf(at.x, (float)(kBins - 1)), fminf(at.y, (float)(kBins - 1))};
            const Two in = add2(at, Two{kWhole, kWhole});
            const Two f = fma2(at, Two{-1.f, -1.f}, add2(in, Two{-kWhole, -kWhole}));
            bin[y] = Row::low(in.x), bin[y + 1] = Row::low(in.y);
            w[y] = share(f.x), w[y + 1] = share(f.y);
          }
#pragma unroll
          for (int y = 0; y < 8; ++y) {
            if (by_k && x[y] >= at_least) atomicAdd(&sh.bins.n[bin[y]], 1u);
            if (by_p && x[y] >= at_least) atomicAdd(&sh.bins.w[bin[y]], (unsigned)w[y]);
          }
        }
        sync();
        all = sum_up(by_k || by_value ? sh.bins.n : nullptr, by_p && !by_value ? sh.bins.w : nullptr, nullptr, kUnit / scale);
        ready = true;
      }
      // (of the two cuts the one that keeps fewer: the bins' weights are rounded otherwise than those that `kept` was summed
      // from, so that top-p's share of them can end behind the k-th id)
      if (weights)
        cut = max(cut, find(from, true, min(by_k ? target_of(kept) : target, all.weight), kept));
      else if ((unsigned)top_k <= all.count)  // (of exactly so many, too: `from` is not asked of every id in the draw)
        cut = find(from, false, top_k, kept);
      else  // (admitted ids of -inf are counted, but not there)
        kept = all.weight;
    }
  }

  // ---- the draw: the largest w / e is the smallest e 2^((m - l) c)
  Pick p = {INFINITY, row.m, INT_MAX, INT_MAX};
  {
    const float last = cut ? logit_of(cut) : -INFINITY;  // the last logit that is kept, and of those ids that have it the last
    const int last_id = cut ? id_of(cut) : INT_MAX;
    float from = last;
    if (min_p > 0.f && row.c2 > 0.f) from = fmaxf(from, row.least(-log2f(min_p) / row.c2));
    from = fmaxf(from, -FLT_MAX);
    const float* noise = s.d_noise + b * s.noise_stride + lo;
    const bool aligned = ((uintptr_t)(noise - pad) & 15) == 0;  // a line's noise is, too
    constexpr int kLines = 16 / N;  // sixteen ids of a thread at once
    int best = 0;  // place of the best id, first line's and its number of the sixteen
    if (top == row.m) {
      const T* x = reinterpret_cast<const T*>(lines + top_v);
      for (int e = N - 1; e >= 0; --e)
        if (value(x[e]) == row.m) p.first = id_at(top_v * N + e - pad);
    }
    for (int v0 = tid; v0 < count_v && !first; v0 += kLines * kThreads) {
      uint4 r[kLines], q[4];
      bool some[kLines];
#pragma unroll
      for (int y = 0; y < kLines; ++y) {
        const int v = v0 + y * kThreads, i = v * N - pad;
        r[y] = lines[min(v, count_v - 1)];
        some[y] = v < count_v && L::top(r[y]) >= from;
        const bool whole = taken < 0 && aligned && lo + i >= 0 && lo + i + N <= s.V;  // (nothing outside the row is read)
#pragma unroll
        for (int e = 0; e < N / 4; ++e) {
          uint4& o = q[y * (N / 4) + e];
          o = make_uint4(0x7F800000u, 0x7F800000u, 0x7F800000u, 0x7F800000u);
          load_if(o, noise + i + 4 * e, some[y] && whole);
          if (some[y] && !whole) {
            float n4[4] = {INFINITY, INFINITY, INFINITY, INFINITY};
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const int k = i + 4 * e + z;
              const bool in = k >= 0 && k < (taken >= 0 ? taken : n);
              load_if(n4[z], noise + (in && taken >= 0 ? (int)places()[k] : k), in);
            }
            o = make_uint4(__float_as_uint(n4[0]), __float_as_uint(n4[1]), __float_as_uint(n4[2]), __float_as_uint(n4[3]));
          }
        }
      }
#pragma unroll
      for (int y = 0; y < kLines; ++y) {
        if (!some[y]) continue;
        // ids of the last logit kept, behind the last one: not kept
        const int i0 = (v0 + y * kThreads) * N - pad;
        if (cut && (taken >= 0 || lo + i0 + N - 1 > last_id)) {
          bool tie = false;
#pragma unroll
          for (int z = 0; z < N; z += 2) {
            const Two x = L::pair(r[y], z / 2);
            tie = tie || x.x == last || x.y == last;
          }
          if (tie)
#pragma unroll
            for (int z = 0; z < N; ++z) {
              const Two x = L::pair(r[y], z / 2);
              if ((z & 1 ? x.y : x.x) == last && id_at(i0 + z) > last_id) {
                uint4& o = q[y * (N / 4) + z / 4];
                (z % 4 == 0 ? o.x : z % 4 == 1 ? o.y : z % 4 == 2 ? o.z : o.w) = 0u;
              }
            }
        }
#pragma unroll
        for (int z = 0; z < N; z += 2) {
          const Two x = L::pair(r[y], z / 2);
          const Two t = mul2(fma2(x, -0.5f, 0.5f * row.m), Two{row.c2, row.c2});
          const uint4 o = q[y * (N / 4) + z / 4];
          const float e0 = __uint_as_float(z % 4 ? o.z : o.x), e1 = __uint_as_float(z % 4 ? o.w : o.y);
          const float s0 = e0 * exp2_fast(t.x), s1 = e1 * exp2_fast(t.y);  // (infinite where the id is not admitted)
          if (e0 >= FLT_MIN && x.x >= from && t.x <= t_most && s0 < p.score) p.score = s0, best = v0 * 16 + y * N + z;
          if (e1 >= FLT_MIN && x.y >= from && t.y <= t_most && s1 < p.score) p.score = s1, best = v0 * 16 + y * N + z + 1;
        }
      }
    }
    if (p.score < INFINITY) {
      const int i = (best / 16 + best % 16 / N * kThreads) * N + best % N;
      p.id = id_at(i - pad);
      p.logit = value(reinterpret_cast<const T*>(lines)[i]);
    }
  }
  // the block's best of all threads
  p = best_warp(p);
  if (lane == 0) sh.picks[warp] = p;
  __syncthreads();
  if (warp == 0) {
    p = best_warp(sh.picks[lane % kWarps]);
    if (lane == 0) {
      put(sh.pick[rank].score, p.score, 0);
      put(sh.pick[rank].id, p.id, 0);
      put(sh.pick[rank].first, p.first, 0);
      put(sh.pick[rank].logit, p.logit, 0);
    }
  }
  sync();
  if (rank == 0 && warp == 0) {
    p = best_warp(sh.pick[lane % blocks]);
    if (lane == 0) write(p.score < INFINITY ? p.id : p.first, p.score < INFINITY ? p.logit : row.m);
  }
}

}  // namespace
}  // namespace grid

using namespace grid;

extern "C" int grid_sample(const grid_sample_step* s, void* stream) {
  if (!s || !s->d_logits || !s->d_noise || !s->d_tokens || !s->d_status || s->B <= 0 || s->V <= 0 ||
      (s->dtype != GRID_DTYPE_F32 && s->dtype != GRID_DTYPE_BF16))
    return set_error(GRID_E_INVALID_ARG, "grid_sample: bad arguments");
  const int size = s->dtype == GRID_DTYPE_F32 ? 4 : 2;
  if (s->logit_stride < 0 || s->mask_stride < 0 || s->noise_stride < 0 || (uintptr_t)s->d_logits % size ||
      (uintptr_t)s->d_mask % 4 || (uintptr_t)s->d_noise % 4)
    return set_error(GRID_E_INVALID_ARG, "grid_sample: negative stride or unaligned pointer");
  if (s->B > 65535 || s->V > kMaxIds)
    return set_error(GRID_E_TOO_LARGE, "grid_sample: more than 65535 rows or 393216 ids");
  // (blocks by the vocabulary alone: a row's sums do not depend on the batch)
  int blocks = 1, log = 0;
  while (blocks < kMaxBlocks && s->V > 2048 * blocks) blocks *= 2, ++log;
  // (where four blocks to an SM, as many as of the bf16 kernel fit, do not take all rows at once, and the rows are few enough to
  // look at all: 256 rows over 151,937 bf16 logits, some greedy, were 86 us instead of 96.  Of the fp32 kernel two fit: 39 to 76
  // rows over so many ids are more than one wave, too, and keep their own order; 64 with top-p take 53 us)
  const bool sorted = s->B * blocks > 608 && s->B <= 2048 && (s->d_temperature || s->d_top_k || s->d_top_p || s->d_min_p);
  const SampleArgs a = {*s, ((s->V + blocks - 1) / blocks + 31) & ~31, sorted};
  const size_t smem = kSharedRoom + (size_t)a.each * size + 32;
  static std::atomic<uint64_t> ready[2][2][4];  // the devices where a kernel has its room in shared memory
  auto go = [&](auto kernel) {
    std::atomic<uint64_t>& done = ready[size == 4][s->d_mask != nullptr][log];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && !(dev < 64 && done.load() >> dev & 1)) {
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 << 10);
      if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev);
    }
    if (e != cudaSuccess) return e;
    return launch_cluster(kernel, dim3((unsigned)(s->B * blocks)), dim3(kThreads), smem, blocks, (cudaStream_t)stream, a);
  };
  auto launch = [&](auto type, auto masked) {
    using T = decltype(type);
    constexpr bool kMasked = decltype(masked)::value;
    return blocks == 1   ? go(k_sample<T, 1, kMasked>)
           : blocks == 2 ? go(k_sample<T, 2, kMasked>)
           : blocks == 4 ? go(k_sample<T, 4, kMasked>)
                         : go(k_sample<T, 8, kMasked>);
  };
  const std::true_type yes;
  const std::false_type no;
  if (size == 4)
    GRID_CUDA(s->d_mask ? launch(0.f, yes) : launch(0.f, no));
  else
    GRID_CUDA(s->d_mask ? launch((uint16_t)0, yes) : launch((uint16_t)0, no));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}
