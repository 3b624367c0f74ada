// Verification of drafted tokens against the masked target distribution, from
// given random numbers (grid_draft_verify).
//
// For row b and position k let l be the logits, A the admitted ids and c =
// log2(e) / T.  With any base the sum s = sum_A 2^((l - base) c) gives
// p(i) = 2^((l_i - base) c) / s.  k_stats computes (base, s) of pieces of every
// position's logits in one pass: per thread a running base, one of the
// admitted logits, within 16 exponents of the largest so far.  The difference
// comes before the product with c everywhere: at T = 1e-6 the roundings of l c
// alone are whole exponents, while (l - base) c is off by 2^-23 of itself
// whatever T is.  The last of a row's blocks joins the pieces and walks the
// acceptance tests u q(x) < p(x) to the first refusal n.
// k_draw draws the next token from position n alone: argmax w_i / e_i needs no
// running sum over the vocabulary, so the order of the additions decides no
// token.
//
// Both kernels are bound by the bytes they read and, in bf16, by the
// instructions for an id; each id's mask bit is looked at first, and 16 bytes of
// logits that hold no admitted id are not read.  256 rows of 5 positions over
// 151,937 ids (bf16, 414 MB read) take 118 us in a graph, 32 rows in fp32 37, one
// row of 3 positions over 512 ids 7.1 (one launch, a chain of dependent loads; a
// call takes 10); low temperatures move the bases more often: 199 at T = 1e-3 for
// the 256 rows.  K = 0, 32 rows over 151,936 ids: 24 in either type.
// A cluster of blocks per row that stops at the first refusal reads less, but its
// positions follow one another: 61 us (32 rows) and 178 us (256 rows).
#include <cfloat>
#include <cmath>
#include <new>

#include "grid_model.cuh"

namespace grid {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxPieces = 64, kMaxParts = 256;  // of one position's logits, of one draw
constexpr int kMaxDraft = 64;
constexpr int kAlone = 4096;  // ids that a row's last block draws from by itself
// Blocks wanted of either kernel.  Of k_stats, what the SMs hold at once (32 rows of 5 positions in fp32: 36.9 us with 5,
// 39.5 with 8); of k_draw, many short ones (256 rows over 151,937 ids: 118 us with 24, 4 more with 12).
constexpr int kBlocksPerSm = 5, kDrawsPerSm = 24;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct alignas(16) Stat {
  float base, s;  // a logit and the sum over the admitted ids of 2^((l - base) c); base -inf: none is admitted
  float m;        // the largest admitted logit and its first id
  int id;
};
__device__ __forceinline__ Stat no_stat() { return Stat{-INFINITY, 0.f, -INFINITY, INT_MAX}; }

// (l - base) c of a clean l.  By halves, since the difference of two logits may be past the type (c is at most half of the
// largest value); and an id of logit -inf has no weight where T is infinite (c = 0) either.
__device__ __forceinline__ float exponent(float l, float base, float c) {
  return l > -INFINITY ? fmaf(0.5f, l, -0.5f * base) * (2.f * c) : -INFINITY;
}
__device__ __forceinline__ void rebase(Stat& x, float base, float c) {
  x.s = x.base > -INFINITY ? x.s * exp2_fast(exponent(x.base, base, c)) : 0.f;
  x.base = base;
}
// The largest of a warp's floats (none a NaN), to every lane: their bits in the order of integers.
__device__ __forceinline__ float max_warp(float x) {
  int i = __float_as_int(x);
  i = __reduce_max_sync(~0u, i ^ (i >> 31 & INT_MAX));
  return __int_as_float(i ^ (i >> 31 & INT_MAX));
}
// The warp's join, to every lane: the largest base first, then one sum.
template <bool kLargest>
__device__ __forceinline__ Stat join_warp(Stat x, float c) {
  const float base = max_warp(x.base);
  if (base > -INFINITY) rebase(x, base, c);
#pragma unroll
  for (int o = 16; o; o >>= 1) x.s += __shfl_xor_sync(~0u, x.s, o);
  if constexpr (kLargest) {
    const float m = max_warp(x.m);
    x.id = __reduce_min_sync(~0u, x.m == m ? x.id : INT_MAX);
    x.m = m;
  }
  return x;
}

// NaN counts as -inf, +inf as the largest finite value.
__device__ __forceinline__ float clean(float l) { return fminf(fmaxf(l, -INFINITY), FLT_MAX); }
// A load where `in` holds, without a branch: as branches, the loads of a loop wait for one another.
__device__ __forceinline__ void load_if(float& x, const float* p, bool in) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\n@p ld.global.nc.L1::no_allocate.f32 %0, [%1];\n}" : "+f"(x) : "l"(p), "r"((int)in));
}
__device__ __forceinline__ void load_if(uint16_t& x, const uint16_t* p, bool in) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\n@p ld.global.nc.L1::no_allocate.u16 %0, [%1];\n}" : "+h"(x) : "l"(p), "r"((int)in));
}
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }  // bf16

// (p is at most 1; the sum of one weight alone may come out a rounding below it)
__device__ __forceinline__ float log_prob(float l, float c, const Stat& x) {
  return fminf((exponent(l, x.base, c) - log2f(x.s)) * kLn2, 0.f);
}

// The row's 1/T (1 for a greedy row) and whether it is greedy.
__device__ __forceinline__ float inv_temp(const grid_draft_step& a, int b, bool& greedy) {
  const float t = a.d_temperature ? a.d_temperature[b] : 1.f;
  greedy = !(t > 0.f);
  return greedy ? 1.f : fminf(1.f / t, FLT_MAX);
}
__device__ __forceinline__ float scale2(float inv) { return fminf(inv * kLog2e, 0.5f * FLT_MAX); }
__device__ __forceinline__ int draft_len(const grid_draft_step& a, int b) {
  return a.d_draft_len ? min(max(a.d_draft_len[b], 0), a.K) : a.K;
}

template <typename T>
__device__ __forceinline__ const T* logits_at(const grid_draft_step& a, int b, int k) {
  return static_cast<const T*>(a.d_logits) + b * a.logit_stride[0] + k * a.logit_stride[1];
}
__device__ __forceinline__ const uint32_t* mask_at(const grid_draft_step& a, int b, int k) {
  return a.d_mask ? a.d_mask + b * a.mask_stride[0] + k * a.mask_stride[1] : nullptr;
}
__device__ __forceinline__ bool admitted(const uint32_t* mask, int id) { return !mask || (mask[id >> 5] >> (id & 31) & 1); }

// One more term of the sum; l is clean.
__device__ __forceinline__ void add(Stat& x, float l, float c) {
  if (!(l > -INFINITY)) return;
  float t = fmaf(0.5f, l, -0.5f * x.base) * (2.f * c);
  if (!(t <= 16.f)) {  // (infinite or no number where no base is set yet)
    rebase(x, l, c);
    t = 0.f;
  }
  x.s += exp2_fast(t);
}
__device__ __forceinline__ void take(Stat& x, float l, int id, float c) {
  l = clean(l);
  add(x, l, c);
  if (l > x.m || (l == x.m && id < x.id)) x.m = l, x.id = id;
}

// A warp's tile is up to 1,024 ids; the mask bits of ids 32 i .. 32 i + 31 of it
// are lane i's word (0 for ids from `hi` on; t0: the tile's first id).
constexpr int kTileIds = 1024;
__device__ __forceinline__ uint32_t tile_word(const uint32_t* mask, int words, int t0, int hi, int lane) {
  const int t = t0 + 32 * lane;
  if (t >= hi) return 0u;
  uint32_t w = ~0u;
  if (mask) {
    const int i = t >> 5, sh = t & 31;
    w = mask[i];
    if (sh) w = __funnelshift_r(w, i + 1 < words ? mask[i + 1] : 0u, sh);
  }
  return hi - t < 32 ? w & ((1u << (hi - t)) - 1u) : w;
}

// 16 bytes of logits as floats
template <typename T, int N>
__device__ __forceinline__ void unpack(const uint4& raw, float (&y)[N]) {
  const uint32_t r[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if constexpr (N == 4) {
      y[e] = __uint_as_float(r[e]);
    } else {
      y[2 * e] = __uint_as_float(r[e] << 16);
      y[2 * e + 1] = __uint_as_float(r[e] & 0xFFFF0000u);
    }
}

// The logits of a tile go through shared memory, 16 bytes at a time to a place
// of the thread's own, kStages - 1 tiles ahead: what is in flight needs no
// registers.  The words of the masks are read a tile before that; lines that
// hold no admitted id are not read.
template <typename T>
struct Staged {
  static constexpr int kVec = 16 / sizeof(T), kSteps = 4, kStages = 2, kIds = kSteps * 32 * kVec;
  uint4 raw[kStages][kSteps][kThreads];
  uint32_t bits[kStages][kThreads];  // a byte per step
};

// N logits one by one: where the base is not set yet or has to move, and where
// a NaN or an infinity is admitted.
template <int N>
struct Values {
  float y[N];
};
template <int N>
__device__ __noinline__ float2 take_each(float base, float s, Values<N> v, float c) {
  Stat x{base, s, 0.f, 0};
#pragma unroll
  for (int e = 0; e < N; ++e) add(x, clean(v.y[e]), c);
  return make_float2(x.base, x.s);
}

// The ids lo .. hi-1 of one position (l + lo on 16 bytes), by a block.
// kLargest: the first largest logit too, which only greedy rows ask for.
template <typename T, bool kLargest>
__device__ __forceinline__ Stat scan(const T* __restrict__ l, const uint32_t* __restrict__ mask, int words, int lo, int hi, float c,
                                     Staged<T>& st) {
  using S = Staged<T>;
  constexpr int kVec = S::kVec, kPerWord = 32 / kVec;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int whole = lo + (hi - lo) / kVec * kVec, tiles = (whole - lo + S::kIds - 1) / S::kIds;
  const int from = lane / kPerWord, shift = lane % kPerWord * kVec;  // this lane's bits of a step: which word, and where
  Stat x = no_stat();
  int at_max = -1;  // where the 16 bytes of the largest logit begin
  uint32_t ahead = tile_word(mask, words, lo + warp * S::kIds, whole, lane);
  const uint32_t place = (uint32_t)__cvta_generic_to_shared(&st.raw[0][0][tid]);
  auto issue = [&](int tile, int stage) {
    if (tile < tiles) {
      const T* src = l + lo + tile * S::kIds + lane * kVec;
      uint32_t all = 0;
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i) {
        const uint32_t bits = __shfl_sync(~0u, ahead, i * kVec + from) >> shift & ((1u << kVec) - 1u);
        all |= bits << (8 * i);
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\n@p cp.async.cg.shared.global [%0], [%1], 16;\n}" ::"r"(
                         place + (uint32_t)((stage * S::kSteps + i) * sizeof(st.raw[0][0]))),
                     "l"(src + i * 32 * kVec), "r"(bits)
                     : "memory");
      }
      st.bits[stage][tid] = all;
      ahead = tile_word(mask, words, lo + (tile + kWarps) * S::kIds, whole, lane);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) issue(warp + i * kWarps, i);
  int stage = 0;
#pragma unroll 1
  for (int tile = warp; tile < tiles; tile += kWarps) {
    issue(tile + (S::kStages - 1) * kWarps, stage ? stage - 1 : S::kStages - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1) : "memory");
    const uint32_t all = st.bits[stage][tid];
#pragma unroll
    for (int i = 0; i < S::kSteps; ++i) {
      const uint32_t bits = all >> (8 * i) & 0xFFu;
      if (!bits) continue;
      const uint4 r = st.raw[stage][i][tid];
      Values<kVec> v;
      unpack<T>(r, v.y);
#pragma unroll
      for (int e = 0; e < kVec; ++e) v.y[e] = bits & (1u << e) ? v.y[e] : -INFINITY;
      if constexpr (kLargest) {
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < kVec; ++e) top = fmaxf(top, v.y[e]);
        top = clean(top);
        if (top > x.m) {
          x.m = top;
          at_max = lo + tile * S::kIds + (i * 32 + lane) * kVec;
        }
      }
      Two t = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        const Two z = mul2(fma2(Two{v.y[e], v.y[e + 1]}, 0.5f, -0.5f * x.base), Two{2.f * c, 2.f * c});
        t = add2(t, Two{exp2_fast(z.x), exp2_fast(z.y)});
      }
      if (t.x + t.y < 1048576.f) {  // (a base is good for terms up to 2^20; no NaN, of a logit or of -inf x 0, is below it)
        x.s += t.x + t.y;
      } else {
        const float2 y = take_each<kVec>(x.base, x.s, v, c);
        x.base = y.x, x.s = y.y;
      }
    }
    if (++stage == S::kStages) stage = 0;
  }
  if (kLargest && at_max >= 0) {  // the largest logit's id, from its 16 bytes again
    for (int e = kVec - 1; e >= 0; --e)
      if (clean(value(l[at_max + e])) == x.m && admitted(mask, at_max + e)) x.id = at_max + e;
  }
  const int i = whole + tid;
  if (i < hi && admitted(mask, i)) take(x, value(l[i]), i, c);
  return x;
}

// The first largest admitted logit of a position, by a warp.
template <typename T>
__device__ __noinline__ int largest(const T* l, const uint32_t* mask, int V) {
  Stat y = no_stat();
  for (int i = threadIdx.x & 31; i < V; i += 32) {
    const float v = clean(value(l[i]));
    if (v > y.m && admitted(mask, i)) y.m = v, y.id = i;
  }
  return join_warp<true>(y, 0.f).id;
}

// Best score so far and the first id that has it.
struct alignas(8) Best {
  float s;
  int id;
};
__device__ __forceinline__ void better(Best& x, float s, int id) {
  if (s > x.s || (s == x.s && id < x.id)) x = Best{s, id};
}
__device__ __forceinline__ Best best_warp(Best x) {  // (scores are not negative: their bits are in their order)
  const unsigned s = __reduce_max_sync(~0u, __float_as_uint(x.s));
  return Best{__uint_as_float(s), __reduce_min_sync(~0u, __float_as_uint(x.s) == s ? x.id : INT_MAX)};
}
// What scores the ids of a row's draw: w / e with w = max(p - q, 0), by an approximate
// reciprocal (two units in the last place: a score is only compared with
// scores).  0 or less, or not finite: the id cannot be drawn.
struct Scorer {
  float c, base, inv_s;
  __device__ __forceinline__ float operator()(float l, float e, float q) const {
    float t = fmaf(0.5f, l, -0.5f * base) * (2.f * c), r;
    if (!(t < 126.f)) t = exponent(clean(l), base, c);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e));
    return fmaxf(fmaf(exp2_fast(t), inv_s, -q), 0.f) * r;
  }
};
__device__ __forceinline__ void keep(Best& z, float s, int id) {
  if (s > z.s && s < INFINITY) z = Best{s, id};
}

// The draw of a row by the target's own weights, by a warp (no residual weight was left).
template <typename T>
__device__ __noinline__ Best draw_whole(Scorer score, const T* l, const uint32_t* mask, const float* e, int V) {
  Best z{0.f, INT_MAX};
  for (int i = threadIdx.x & 31; i < V; i += 32)
    if (admitted(mask, i)) keep(z, score(value(l[i]), e[i], 0.f), i);
  return best_warp(z);
}

// What a draw needs to know of its row.
struct alignas(16) Row {
  int n;           // position to draw from, or -1: the row's outcome is written
  int out;         // id that the residual leaves out, or -1
  float base, s;
  float c;
  int refused, pad[2];
};

// The best of the ids lo .. hi-1 of row b's draw, by a block; warp 0 gets it.  A
// warp takes 256 ids at a time, a lane per id of eight mask words.
template <typename T>
__device__ __forceinline__ Best draw_part(const grid_draft_step& a, int b, const Row& r, int lo, int hi) {
  constexpr int kWords = 8, kIds = kWords * 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, words = (a.V + 31) / 32;
  __shared__ Best sh[kWarps];
  const Scorer score{r.c, r.base, 1.f / r.s};
  const T* l = logits_at<T>(a, b, r.n);
  const uint32_t* mask = mask_at(a, b, r.n);
  const float* q = r.refused && a.d_probs ? a.d_probs + b * a.prob_stride[0] + r.n * a.prob_stride[1] : nullptr;
  const float* e = a.d_noise + b * a.noise_stride;
  auto word_at = [&](int t0) {
    const uint32_t w = lane < kWords ? tile_word(mask, words, t0, hi, lane) : 0u;
    return (unsigned)(r.out - t0 - 32 * lane) < 32u ? w & ~(1u << (r.out - t0 - 32 * lane)) : w;
  };
  Best z{0.f, INT_MAX};
  uint32_t ahead = word_at(lo + warp * kIds);
#pragma unroll 1
  for (int t0 = lo + warp * kIds; t0 < hi; t0 += kWarps * kIds) {
    const uint32_t word = ahead;
    ahead = word_at(t0 + kWarps * kIds);
    if (!__any_sync(~0u, word != 0)) continue;
    T lv[kWords];
    float ev[kWords], qv[kWords];
#pragma unroll
    for (int u = 0; u < kWords; ++u) {
      const bool in = __shfl_sync(~0u, word, u) >> lane & 1;
      const int id = t0 + 32 * u + lane;
      lv[u] = 0, ev[u] = INFINITY, qv[u] = 0.f;  // (infinite noise: a score of zero)
      load_if(lv[u], l + id, in);
      load_if(ev[u], e + id, in);
      load_if(qv[u], q + id, in && q);
    }
#pragma unroll
    for (int u = 0; u < kWords; ++u) keep(z, score(value(lv[u]), ev[u], qv[u]), t0 + 32 * u + lane);
  }
  z = best_warp(z);
  if (lane == 0) sh[warp] = z;
  __syncthreads();
  return best_warp(lane < kWarps ? sh[lane] : Best{0.f, INT_MAX});
}
// The token that the row's best id makes, by a warp.
template <typename T>
__device__ __forceinline__ void draw_end(const grid_draft_step& a, int b, const Row& r, Best z) {
  const T* l = logits_at<T>(a, b, r.n);
  const uint32_t* mask = mask_at(a, b, r.n);
  if (!(z.s > 0.f) && r.refused)
    z = draw_whole(Scorer{r.c, r.base, 1.f / r.s}, l, mask, a.d_noise + b * a.noise_stride, a.V);
  const int token = z.s > 0.f ? z.id : largest(l, mask, a.V);  // (the latter: no noise was positive)
  if ((threadIdx.x & 31) == 0) {
    a.d_tokens[(size_t)b * (a.K + 1) + r.n] = token;
    if (a.d_logprob)
      a.d_logprob[(size_t)b * (a.K + 1) + r.n] = log_prob(clean(value(l[token])), r.c, Stat{r.base, r.s, 0.f, 0});
    if (token == a.eos) a.d_status[b] = GRID_ST_COMPLETE;
  }
}

// What the tests need of a drafted id.
struct alignas(16) Drafted {
  float l, uq;  // its logit (-inf: refused whatever u is) and u q(x)
  int id, pad;
};
// One piece of one position: block (position row) * pieces + piece.  Pieces
// are cut where the position's 16-byte lines begin, so that rows of any
// alignment are read in whole lines; the ids before the first line belong to
// piece 0, those after the last to the last piece.  The last block of a row
// walks its acceptance tests and writes what they decide; over a small
// vocabulary (kDraws) it also draws, which saves a launch.
template <typename T, bool kDraws>
__global__ void __launch_bounds__(kThreads) k_stats(const grid_draft_step a, Stat* __restrict__ stats, int pieces,
                                                    int piece, int* __restrict__ done, Drafted* __restrict__ drafted,
                                                    Row* __restrict__ rows) {
  const int row = blockIdx.x / pieces, pc = blockIdx.x - row * pieces;
  const int b = row / (a.K + 1), k = row - b * (a.K + 1);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  extern __shared__ __align__(16) uint8_t staged[];
  __shared__ Stat sh[kWarps];
  __shared__ int last;
  Staged<T>& st = *reinterpret_cast<Staged<T>*>(staged);
  pdl_wait();
  pdl_next();
  const int nd = draft_len(a, b);
  if (k > nd) return;
  bool greedy;
  const float c = scale2(inv_temp(a, b, greedy));
  {
    const T* l = logits_at<T>(a, b, k);
    const uint32_t* mask = mask_at(a, b, k);
    if (pc == 0 && k < nd && tid == kThreads - 1) {
      Drafted x{-INFINITY, 0.f, a.d_draft[(size_t)b * a.K + k], 0};
      if (x.id >= 0 && x.id < a.V) {
        const bool in = admitted(mask, x.id);
        const float v = clean(value(l[x.id])), u = a.d_u[(size_t)b * a.K + k];
        const float q = a.d_probs ? a.d_probs[b * a.prob_stride[0] + k * a.prob_stride[1] + x.id] : 1.f;
        if (in) x.l = v, x.uq = u * q;
      }
      drafted[(size_t)b * a.K + k] = x;
      __threadfence();
    }
    const int head = min(a.V, (int)((16 - ((uintptr_t)l & 15)) & 15) / (int)sizeof(T)), words = (a.V + 31) / 32;
    const long long from = (long long)head + (long long)pc * piece;
    const int lo = (int)min((long long)a.V, from), hi = (int)min((long long)a.V, from + piece);
    Stat x = greedy ? scan<T, true>(l, mask, words, lo, hi, c, st) : scan<T, false>(l, mask, words, lo, hi, c, st);
    if (pc == 0 && tid < head && admitted(mask, tid)) take(x, value(l[tid]), tid, c);
    x = join_warp<true>(x, c);
    if (lane == 0) sh[warp] = x;
  }
  __syncthreads();
  if (warp == 0) {
    const Stat x = join_warp<true>(lane < kWarps ? sh[lane] : no_stat(), c);
    if (lane == 0) {
      stats[(size_t)row * pieces + pc] = x;
      __threadfence();
      last = atomicAdd(&done[b], 1) == (nd + 1) * pieces - 1;
      if (last) done[b] = 0;
      __threadfence();
    }
  }
  __syncthreads();
  if (!last) return;
  // ---- the row's acceptance tests
  __shared__ Stat at[kMaxDraft + 1];
  __shared__ int ok[kMaxDraft + 1], ids[kMaxDraft];
  __shared__ float lp[kMaxDraft];
  for (int j = warp; j <= nd; j += kWarps) {
    const Stat* src = stats + ((size_t)b * (a.K + 1) + j) * pieces;
    float4 d = {};
    if (j < nd) d = __ldcg(reinterpret_cast<const float4*>(drafted + (size_t)b * a.K + j));
    float4 y = {-INFINITY, 0.f, -INFINITY, __int_as_float(INT_MAX)};
    if (lane < pieces) y = __ldcg(reinterpret_cast<const float4*>(src + lane));
    Stat x = join_warp<true>(Stat{y.x, y.y, y.z, __float_as_int(y.w)}, c);
    for (int i = 32; i < pieces; i += 32) {
      Stat z = no_stat();
      if (i + lane < pieces) {
        y = __ldcg(reinterpret_cast<const float4*>(src + i + lane));
        z = Stat{y.x, y.y, y.z, __float_as_int(y.w)};
      }
      z = join_warp<true>(z, c);
      x = join_warp<true>(lane == 0 ? x : lane == 1 ? z : no_stat(), c);
    }
    if (lane == 0) {
      at[j] = x;
      ok[j] = 0;
      if (j < nd) {
        const int id = ids[j] = __float_as_int(d.z);
        if (d.x > -INFINITY) {
          ok[j] = greedy ? id == x.id : d.y < exp2_fast(exponent(d.x, x.base, c)) / x.s;
          if (ok[j] && id == a.eos) ok[j] = 2;
          lp[j] = log_prob(d.x, c, x);
        }
      }
    }
  }
  __syncthreads();
  int n = 0;
  bool ended = false;
  while (n < nd && ok[n] && !ended) ended = ok[n++] == 2;
  const Stat x = at[min(n, nd)];
  const bool empty = !ended && !(x.base > -INFINITY);
  const bool settled = ended || empty || greedy;
  for (int j = tid; j <= a.K; j += kThreads) {
    const int id = j < n ? ids[j] : j == n && !ended && !empty && greedy ? x.id : -1;
    a.d_tokens[(size_t)b * (a.K + 1) + j] = id;
    if (a.d_logprob) a.d_logprob[(size_t)b * (a.K + 1) + j] = j < n ? lp[j] : id >= 0 ? log_prob(x.m, c, x) : 0.f;
  }
  const Row r{settled ? -1 : n, n < nd && !a.d_probs ? ids[n] : -1, x.base, x.s, c, n < nd, {0, 0}};
  if (tid == 0) {
    a.d_accepted[b] = n;
    a.d_status[b] = ended || (!empty && greedy && x.id == a.eos) ? GRID_ST_COMPLETE : empty ? GRID_ST_EMPTY_MASK : GRID_ST_OK;
    if (!kDraws) rows[b] = r;
  }
  if (kDraws && !settled) {
    const Best z = draw_part<T>(a, b, r, 0, a.V);  // (its barrier lies between what was written above and the token)
    if (warp == 0) draw_end<T>(a, b, r, z);
  }
}

// The draw of one row: block row * parts + part scores its part of the
// vocabulary at the row's position n; the last of the row's blocks writes the
// token.
template <typename T>
__global__ void __launch_bounds__(kThreads, 5) k_draw(const grid_draft_step a, const Row* __restrict__ rows,
                                                      Best* __restrict__ best, int* __restrict__ done, int parts, int part) {
  const int b = blockIdx.x / parts, pt = blockIdx.x - b * parts, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_next();
  const float4* row = reinterpret_cast<const float4*>(rows + b);
  const float4 r4 = __ldcg(row), s4 = __ldcg(row + 1);
  const Row r{__float_as_int(r4.x), __float_as_int(r4.y), r4.z, r4.w, s4.x, __float_as_int(s4.y), {0, 0}};
  if (r.n < 0) return;
  const int lo = min(a.V, pt * part);
  Best z = draw_part<T>(a, b, r, lo, min(a.V, lo + part));
  if (threadIdx.x >= 32) return;
  int last = 0;
  if (lane == 0) {
    best[(size_t)b * parts + pt] = z;
    __threadfence();
    last = atomicAdd(&done[b], 1) == parts - 1;
    if (last) done[b] = 0;
    __threadfence();
  }
  if (!__shfl_sync(~0u, last, 0)) return;
  z = Best{0.f, INT_MAX};
  for (int i = lane; i < parts; i += 32) {
    const float2 y = __ldcg(reinterpret_cast<const float2*>(best + (size_t)b * parts + i));
    better(z, y.x, __float_as_int(y.y));
  }
  draw_end<T>(a, b, r, best_warp(z));
}

}  // namespace
}  // namespace grid

using namespace grid;

struct grid_drafts {
  int B = 0, K = 0, V = 0, sms = 152;
  Stat* stats = nullptr;
  Best* best = nullptr;
  Row* rows = nullptr;
  Drafted* drafted = nullptr;
  int* done = nullptr;
  Arena mem;
};

extern "C" int grid_drafts_create(int32_t B, int32_t K, int32_t V, grid_drafts** out) {
  if (!out || B <= 0 || K < 0 || K > kMaxDraft || V <= 0)
    return set_error(GRID_E_INVALID_ARG, "grid_drafts_create: B and V are positive, K in 0 .. 64");
  if (B > 65535 || V > (1 << 30))
    return set_error(GRID_E_TOO_LARGE, "grid_drafts_create: more than 65535 rows or 2^30 ids");
  grid_drafts* d = new (std::nothrow) grid_drafts;
  if (!d) return set_error(GRID_E_TOO_LARGE, "grid_drafts_create: out of host memory");
  d->B = B;
  d->K = K;
  d->V = V;
  int rc = GRID_OK, dev = 0;
  cudaError_t e = cudaSuccess;
  auto room = [](auto kernel, size_t bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  };
  // (a call cuts n positions into at most n + kBlocksPerSm * sms pieces)
  if ((e = cudaGetDevice(&dev)) == cudaSuccess &&
      (e = cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, dev)) == cudaSuccess &&
      !(rc = d->mem.alloc(((size_t)B * (K + 1) + kBlocksPerSm * d->sms) * sizeof(Stat), (void**)&d->stats)) &&
      !(rc = d->mem.alloc((size_t)B * kMaxParts * sizeof(Best), (void**)&d->best)) &&
      !(rc = d->mem.alloc((size_t)B * sizeof(Row), (void**)&d->rows)) &&
      !(rc = d->mem.alloc((size_t)B * K * sizeof(Drafted), (void**)&d->drafted)) &&
      !(rc = d->mem.alloc((size_t)B * sizeof(int), (void**)&d->done)) &&
      (e = cudaMemset(d->done, 0, (size_t)B * sizeof(int))) == cudaSuccess &&
      (e = room(k_stats<float, false>, sizeof(Staged<float>))) == cudaSuccess &&
      (e = room(k_stats<float, true>, sizeof(Staged<float>))) == cudaSuccess &&
      (e = room(k_stats<uint16_t, false>, sizeof(Staged<uint16_t>))) == cudaSuccess &&
      (e = room(k_stats<uint16_t, true>, sizeof(Staged<uint16_t>))) == cudaSuccess)
    e = cudaDeviceSynchronize();
  if (rc || e != cudaSuccess) {
    d->mem.release();
    delete d;
    return rc ? rc : set_error(GRID_E_CUDA, std::string("grid_drafts_create: ") + cudaGetErrorString(e));
  }
  *out = d;
  return GRID_OK;
}

extern "C" void grid_drafts_free(grid_drafts* d) {
  if (!d) return;
  d->mem.release();
  delete d;
}

extern "C" int grid_draft_verify(const grid_drafts* d, const grid_draft_step* s, void* stream) {
  if (!d || !s || !s->d_logits || !s->d_noise || !s->d_tokens || !s->d_accepted || !s->d_status || s->B <= 0 ||
      s->K < 0 || s->V <= 0 || (s->K && (!s->d_draft || !s->d_u)) ||
      (s->dtype != GRID_DTYPE_F32 && s->dtype != GRID_DTYPE_BF16))
    return set_error(GRID_E_INVALID_ARG, "grid_draft_verify: bad arguments");
  if (s->B > d->B || s->K > d->K || s->V > d->V)
    return set_error(GRID_E_TOO_LARGE, "grid_draft_verify: B, K or V is larger than the handle's");
  const int size = s->dtype == GRID_DTYPE_F32 ? 4 : 2;
  if (s->logit_stride[0] < 0 || s->logit_stride[1] < 0 || s->mask_stride[0] < 0 || s->mask_stride[1] < 0 ||
      s->prob_stride[0] < 0 || s->prob_stride[1] < 0 || s->noise_stride < 0 || (uintptr_t)s->d_logits % size ||
      (uintptr_t)s->d_mask % 4 || (uintptr_t)s->d_probs % 4 || (uintptr_t)s->d_noise % 4)
    return set_error(GRID_E_INVALID_ARG, "grid_draft_verify: negative stride or unaligned pointer");
  // Pieces of a position and parts of a draw: blocks for every SM, none of them of less than a tile for each of its warps.
  auto cut = [&](long long rows, long long per_sm, int least, int most, int& count, int& size_) {
    const long long want = std::min<long long>((per_sm * d->sms + rows - 1) / rows, most);
    size_ = (int)std::max<long long>(least, (s->V + want - 1) / want);
    size_ = (size_ + kTileIds - 1) / kTileIds * kTileIds;
    count = (s->V + size_ - 1) / size_;
  };
  const long long rows = (long long)s->B * (s->K + 1);
  int pieces, piece, parts, part;
  cut(rows, kBlocksPerSm, kWarps * kTileIds, kMaxPieces, pieces, piece);
  // (a warp draws from twice 256 ids, or once where the SMs would not all have a block: 32 rows over 151,936 ids take 36.9 us
  // so and 40.1 with one; 8 rows over 32,000 14.6 and 13.8)
  const bool few = (long long)s->B * s->V < 4LL * kTileIds * d->sms;
  cut(s->B, kDrawsPerSm, (few ? 2 : 4) * kTileIds, kMaxParts, parts, part);
  const bool alone = s->V <= kAlone;
  auto go = [&](auto stats, auto draw, size_t staged) {
    cudaError_t e = launch_pdl(stats, dim3((unsigned)(rows * pieces)), dim3(kThreads), staged, (cudaStream_t)stream, *s, d->stats,
                               pieces, piece, d->done, d->drafted, d->rows);
    if (e != cudaSuccess || alone) return e;
    return launch_pdl(draw, dim3((unsigned)(s->B * parts)), dim3(kThreads), 0, (cudaStream_t)stream, *s, (const Row*)d->rows,
                      d->best, d->done, parts, part);
  };
  using H = uint16_t;
  if (size == 4)
    GRID_CUDA(alone ? go(k_stats<float, true>, k_draw<float>, sizeof(Staged<float>))
                    : go(k_stats<float, false>, k_draw<float>, sizeof(Staged<float>)));
  else
    GRID_CUDA(alone ? go(k_stats<H, true>, k_draw<H>, sizeof(Staged<H>)) : go(k_stats<H, false>, k_draw<H>, sizeof(Staged<H>)));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}
