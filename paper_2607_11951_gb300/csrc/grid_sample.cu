// Sampling from a masked distribution cut by top-k, top-p and min-p, from given
// random numbers (grid_sample).
//
// With m the row's largest admitted logit and c = log2(e) / T, an id's weight is
// w = 2^((l - m) c), its probability w / Z with Z the sum over the admitted ids.
// Ids are ordered by one 54-bit number, the logit's bits in the order of integers
// and then the id's complement, so that what top-k and top-p keep is "order >=
// X".  X is found by counting: the ids of the present range go into 1,024 bins
// that keep the order (of the first level by m - l, linearly; of later ones by
// the order itself), with the number and the weight of each; the bin is found
// in which the k-th id, or top_p of the weight, is reached; and if it holds few
// enough ids, these are sorted and X is one of them, else the bin is the next
// level's range.  Each later level takes ten bits off the order: six at most.
//
// Weights are added as integers, in steps of 2^-40 of the largest, so that their
// sums do not depend on the order of the atomic additions (V ids are off by V
// 2^-41 of the largest weight at most, less than by the rounding of w itself).
//
// A cluster of blocks per row holds the row's admitted logits in its shared
// memory: each logit is read from memory once, noise only where an id is kept.
#include <atomic>
#include <cfloat>
#include <climits>
#include <cmath>

#include "grid_model.cuh"

namespace grid {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxBlocks = 8;             // of a row: the largest cluster that every device takes
constexpr int kBins = 1024, kBinBits = 10;
constexpr int kList = 1024;               // ids that are sorted at once
constexpr int kIdBits = 22;
constexpr int kMaxIds = 393216;           // 48 Ki fp32 logits for each of eight blocks
constexpr float kFirstRange = 40.f;       // exponents below m that the first level's bins reach, or to the smallest logit
constexpr float kUnit = 1099511627776.f;  // 2^40
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
using u64 = unsigned long long;

struct SampleArgs {
  grid_sample_step s;
  int blocks, each;  // blocks of a row, ids of a block (a multiple of 32)
};

struct Pick {   // of a draw: the best score, its id and logit; the first id of the largest logit
  float score, logit;
  int id, first;
};
struct Found {  // the bin that a search ends in, and what lies in the bins before it
  int bin;
  unsigned count;
  u64 weight;
};

struct Hist {
  unsigned n[kBins], lo[kBins], hi[kBins];  // ids, and the two halves of their weights
};
struct Shared {
  union {
    Hist hist;
    u64 list[kList];
  };
  float top, low, z;           // this block's largest and smallest admitted logit, and its weights
  unsigned part_n[2];          // of this block's share of the bins: of the first level, of a later one
  u64 part_w[2];
  u64 most, least;             // of this block's ids in the present bin
  unsigned listed;             // block 0: how many ids the list got
  u64 cut, kept;               // X, and the weight of what it keeps
  Found found;
  Pick pick[kMaxBlocks];       // block 0: of every block
  float zs[kMaxBlocks];
  u64 sums[kWarps], sums2[kWarps];
  Pick picks[kWarps];
  float zw[kWarps];
};
constexpr int kSharedRoom = (sizeof(Shared) + 127) & ~127;

__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
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
__device__ __forceinline__ unsigned get(const unsigned& x, int r) {
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(there(&x, r)) : "memory");
  return v;
}
__device__ __forceinline__ float get(const float& x, int r) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there(&x, r)) : "memory");
  return v;
}
__device__ __forceinline__ u64 get(const u64& x, int r) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(there(&x, r)) : "memory");
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

__device__ __forceinline__ u64 shfl_xor(u64 x, int o) { return __shfl_xor_sync(~0u, x, o); }
__device__ __forceinline__ u64 max_warp(u64 x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = max(x, shfl_xor(x, o));
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
  if (y.score > x.score || (y.score == x.score && y.id < x.id)) x.score = y.score, x.logit = y.logit, x.id = y.id;
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

// A logit as it is kept: NaN as -inf, +inf as the largest finite value of its type, -0 as 0.
__device__ __forceinline__ float kept_as(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX) + 0.f; }
__device__ __forceinline__ uint16_t kept_as(uint16_t x) {  // bf16
  if ((x & 0x7FFF) > 0x7F80) return 0xFF80;
  return x == 0x7F80 ? 0x7F7F : x == 0x8000 ? 0 : x;
}
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <typename T>
__device__ __forceinline__ T nothing();
template <>
__device__ __forceinline__ float nothing<float>() { return -INFINITY; }
template <>
__device__ __forceinline__ uint16_t nothing<uint16_t>() { return 0xFF80; }

// The logit's bits in the order of integers, then the id's complement; and back.
__device__ __forceinline__ u64 order_of(float x, int id) {
  const unsigned b = __float_as_uint(x);
  return (u64)(b ^ ((unsigned)((int)b >> 31) | 0x80000000u)) << kIdBits | (unsigned)((1 << kIdBits) - 1 - id);
}
__device__ __forceinline__ float logit_of(u64 o) {
  const unsigned k = (unsigned)(o >> kIdBits);
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// What a row asks for.
struct Row {
  float c2;        // 2 log2(e) / T
  float m, by;     // the largest logit; bins per half of m - l
  bool first;      // only the first id is kept
  // half of m - l: of the halves, since the difference of two logits may be past the type
  __device__ __forceinline__ float below(float x) const { return fmaf(0.5f, m, -0.5f * x); }
  __device__ __forceinline__ float weight(float x) const { return exp2_fast(-below(x) * c2); }
  __device__ __forceinline__ int bin(float x) const { return (int)fminf(below(x) * by, (float)(kBins - 1)); }
};
__device__ __forceinline__ u64 units(float w) { return __float2ull_rn(w * kUnit); }

template <typename T>
__global__ void __launch_bounds__(kThreads) k_sample(const SampleArgs a) {
  extern __shared__ __align__(128) uint8_t raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  // bins of this block's share, added up over the row's blocks and from the first one of the share on: of the first level, of a later one
  const int share = kBins / a.blocks;
  unsigned* const tot_n = reinterpret_cast<unsigned*>(raw + kSharedRoom);
  u64* const tot_w = reinterpret_cast<u64*>(tot_n + 2 * share);
  T* const vals = reinterpret_cast<T*>(tot_w + 2 * share);
  const grid_sample_step& s = a.s;
  const int b = blockIdx.x / a.blocks, rank = cluster_rank(), blocks = a.blocks;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lo = min(s.V, rank * a.each), n = min(s.V, lo + a.each) - lo;
  pdl_wait();
  // ---- the block's logits, admitted ones as they are and the others as -inf
  Row row;
  const float temp = s.d_temperature ? s.d_temperature[b] : 1.f;
  const int top_k = s.d_top_k ? s.d_top_k[b] : 0;
  const float top_p = s.d_top_p ? s.d_top_p[b] : 1.f, min_p = s.d_min_p ? s.d_min_p[b] : 0.f;
  const bool greedy = !(temp > 0.f);
  row.first = greedy || top_k == 1 || top_p <= 0.f || min_p > 1.f;
  row.c2 = fminf((greedy ? 1.f : 1.f / temp) * (2.f * kLog2e), FLT_MAX);
  float top = -INFINITY, low = INFINITY;
  {
    const T* l = static_cast<const T*>(s.d_logits) + b * s.logit_stride + lo;
    const uint32_t* mask = s.d_mask ? s.d_mask + b * s.mask_stride + (lo >> 5) : nullptr;
    for (int i = tid; i < n; i += kThreads) {  // (a warp's ids are those of one word: lo is a multiple of 32)
      T x = nothing<T>();
      if (!mask || (mask[i >> 5] >> (i & 31) & 1u)) x = kept_as(l[i]);
      vals[i] = x;
      const float v = value(x);
      top = fmaxf(top, v);
      if (v > -INFINITY) low = fminf(low, v);
    }
  }
  // what every thread has, over the block, to a place of sh
  auto over_block = [&](float x, float y) {
    x = max_warp(x), y = max_warp(y);
    if (lane == 0) sh.sums[warp] = (u64)__float_as_uint(x) << 32 | __float_as_uint(y);
    __syncthreads();
    const u64 v = sh.sums[lane % kWarps];
    x = max_warp(__uint_as_float((unsigned)(v >> 32))), y = max_warp(__uint_as_float((unsigned)v));
    if (tid == 0) sh.top = x, sh.low = y;
  };
  over_block(top, -low);
  cluster_sync();
  top = max_warp(lane < blocks ? get(sh.top, lane) : -INFINITY);
  low = -max_warp(lane < blocks ? get(sh.low, lane) : -INFINITY);
  if (!(top > -INFINITY)) {  // (the same in every block)
    if (rank == 0 && tid == 0) {
      s.d_tokens[b] = -1;
      if (s.d_logprob) s.d_logprob[b] = 0.f;
      s.d_status[b] = GRID_ST_EMPTY_MASK;
    }
    cluster_sync();
    return;
  }
  row.m = top;
  {
    const float range = fminf(kFirstRange / row.c2, row.below(low));
    row.by = range > 0.f ? fminf(kBins / range, FLT_MAX) : 0.f;
  }

  // ---- the range of order that is looked at: everything, a bin of the first level, [least, most]
  const bool by_k = !row.first && top_k > 0 && top_k < s.V, by_p = !row.first && top_p < 1.f;
  u64 most = ~0ull, least = 0, cut = 0;
  int first_bin = -1, shift = 0;  // -1: everything
  auto in_range = [&](float x, int i) {
    if (first_bin >= 0) return row.bin(x) == first_bin;
    const u64 o = order_of(x, lo + i);
    return o >= least && o <= most;
  };
  // the range's ids into bins
  auto count = [&](bool level0, bool counts, bool weights) {
    for (int i = tid; i < kBins; i += kThreads) sh.hist.n[i] = sh.hist.lo[i] = sh.hist.hi[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const float x = value(vals[i]);
      if (!(x > -INFINITY)) continue;
      int bin;
      if (level0) {
        bin = row.bin(x);
      } else {
        const u64 o = order_of(x, lo + i);
        if (o < least || o > most) continue;
        bin = (int)((most - o) >> shift);
      }
      if (counts) atomicAdd(&sh.hist.n[bin], 1u);
      if (weights) {
        const u64 w = units(row.weight(x));
        const unsigned l = (unsigned)w, was = l ? atomicAdd(&sh.hist.lo[bin], l) : 0u;
        const unsigned h = (unsigned)(w >> 32) + (was + l < was);
        if (h) atomicAdd(&sh.hist.hi[bin], h);
      }
    }
    cluster_sync();
    // a thread per bin of the block's share (several where the share is large), then the sums from its first bin on
    unsigned* const tn = tot_n + (level0 ? 0 : share);
    u64* const tw = tot_w + (level0 ? 0 : share);
    unsigned base_n = 0;
    u64 base_w = 0;
    for (int j0 = 0; j0 < share; j0 += kThreads) {
      const int j = j0 + tid;
      u64 cn = 0, cw = 0;
      if (j < share)
        for (int r = 0; r < blocks; ++r) {
          const int bin = rank * share + j;
          cn += get(sh.hist.n[bin], r);
          cw += (u64)get(sh.hist.lo[bin], r) + ((u64)get(sh.hist.hi[bin], r) << 32);
        }
      // inclusive sums over the block's threads
      for (int o = 1; o < 32; o <<= 1) {
        const u64 x = __shfl_up_sync(~0u, cn, o), y = __shfl_up_sync(~0u, cw, o);
        if (lane >= o) cn += x, cw += y;
      }
      if (lane == 31) sh.sums[warp] = cn, sh.sums2[warp] = cw;
      __syncthreads();
      u64 all_n = 0, all_w = 0;
      for (int x = 0; x < kWarps; ++x) {
        if (x < warp) cn += sh.sums[x], cw += sh.sums2[x];
        all_n += sh.sums[x], all_w += sh.sums2[x];
      }
      if (j < share) tn[j] = base_n + (unsigned)cn, tw[j] = base_w + cw;
      base_n += (unsigned)all_n, base_w += all_w;
      __syncthreads();
    }
    if (tid == 0) sh.part_n[!level0] = base_n, sh.part_w[!level0] = base_w;
    cluster_sync();
  };
  // the bin in which, after `before`, the target is reached
  auto search = [&](bool level0, bool weights, u64 target, const Found& before) {
    const unsigned* const tn = tot_n + (level0 ? 0 : share);
    const u64* const tw = tot_w + (level0 ? 0 : share);
    unsigned fn = before.count;
    u64 fw = before.weight;
    for (int r = 0; r < rank; ++r) fn += get(sh.part_n[!level0], r), fw += get(sh.part_w[!level0], r);
    for (int j = tid; j < share; j += kThreads) {
      const unsigned pn = fn + (j ? tn[j - 1] : 0);
      const u64 pw = fw + (j ? tw[j - 1] : 0);
      const u64 prev = weights ? pw : pn, now = weights ? fw + tw[j] : fn + tn[j];
      if (prev < target && now >= target)
        for (int r = 0; r < blocks; ++r) {
          put(sh.found.bin, rank * share + j, r);
          put(sh.found.count, pn, r);
          put(sh.found.weight, pw, r);
        }
    }
    cluster_sync();
    return sh.found;
  };
  // X of a target: the least order that is kept; `kept`: the weight of what it keeps
  auto find = [&](bool weights, u64 target, bool want_weight, u64& kept) {
    Found f = search(true, weights, target, Found{0, 0u, 0ull});
    first_bin = f.bin;
    for (;;) {
      // the bin's ids: the first and the last, and a list of them in block 0
      if (tid == 0) sh.listed = 0;
      cluster_sync();
      u64 hi = 0, lo_c = 0;  // (the smallest as the largest complement)
      for (int i = tid; i < n; i += kThreads) {
        const float x = value(vals[i]);
        if (!(x > -INFINITY) || !in_range(x, i)) continue;
        const u64 o = order_of(x, lo + i);
        hi = max(hi, o), lo_c = max(lo_c, ~o);
        unsigned at;
        asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(at) : "r"(there(&sh.listed, 0)) : "memory");
        if (at < kList) put(sh.list[at], o, 0);
      }
      hi = max_warp(hi), lo_c = max_warp(lo_c);
      if (lane == 0) sh.sums[warp] = hi, sh.sums2[warp] = lo_c;
      __syncthreads();
      hi = max_warp(sh.sums[lane % kWarps]), lo_c = max_warp(sh.sums2[lane % kWarps]);
      if (tid == 0) sh.most = hi, sh.least = lo_c;
      cluster_sync();
      const unsigned listed = get(sh.listed, 0);
      most = max_warp(lane < blocks ? get(sh.most, lane) : 0ull);
      least = ~max_warp(lane < blocks ? get(sh.least, lane) : 0ull);
      first_bin = -1;
      if (listed <= kList) {
        if (rank == 0) {
          // ---- sorted, the largest first; the sums of their weights
          int size = 32;
          while (size < (int)listed) size *= 2;
          for (int i = listed + tid; i < size; i += kThreads) sh.list[i] = 0;
          __syncthreads();
          for (int k = 2; k <= size; k *= 2)
            for (int j = k / 2; j; j /= 2) {
              for (int x = tid; x < size / 2; x += kThreads) {
                const int i = 2 * x - (x & (j - 1)), y = i + j;
                const u64 p = sh.list[i], q = sh.list[y];
                if ((p < q) == !(i & k)) sh.list[i] = q, sh.list[y] = p;
              }
              __syncthreads();
            }
          u64 before = f.weight;
          for (int i0 = 0; i0 < size; i0 += kThreads) {
            const int i = i0 + tid;
            const bool some = i < (int)listed;
            const u64 w = some && (weights || want_weight) ? units(row.weight(logit_of(sh.list[i]))) : 0;
            u64 pre = w;
            for (int o = 1; o < 32; o <<= 1) {
              const u64 x = __shfl_up_sync(~0u, pre, o);
              if (lane >= o) pre += x;
            }
            if (lane == 31) sh.sums[warp] = pre;
            __syncthreads();
            u64 all = 0;
            for (int x = 0; x < kWarps; ++x) {
              if (x < warp) pre += sh.sums[x];
              all += sh.sums[x];
            }
            // the last one kept: the target is not reached before it, and is with it
            const u64 prev = weights ? before + pre - w : f.count + (u64)i, now = weights ? before + pre : f.count + (u64)i + 1;
            if (some && prev < target && now >= target)
              for (int r = 0; r < blocks; ++r) {
                put(sh.cut, sh.list[i], r);
                put(sh.kept, before + pre, r);
              }
            before += all;
            __syncthreads();
          }
        }
        cluster_sync();
        kept = sh.kept;
        return sh.cut;
      }
      // ---- the next level
      const int bits = 64 - __clzll((long long)(most - least));
      shift = max(0, bits - kBinBits);
      count(false, !weights, weights || want_weight);
      const Found g = search(false, weights, target, f);
      most -= (u64)g.bin << shift;
      if (most - least >> shift) least = most - ((1ull << shift) - 1);
      f = g;
    }
  };

  // ---- the weights' sum, and the first level's bins
  float z = 0.f;
  for (int i = tid; i < n; i += kThreads) {
    const float x = value(vals[i]);
    if (x > -INFINITY) z += row.weight(x);  // (-inf has no weight where T is infinite either)
  }
  z = sum_warp(z);
  if (lane == 0) sh.zw[warp] = z;
  __syncthreads();
  if (tid == 0) {
    z = 0.f;
    for (int x = 0; x < kWarps; ++x) z += sh.zw[x];
    put(sh.zs[rank], z, 0);
  }
  if (by_k || by_p) {
    count(true, true, by_p);
    unsigned all_n = 0;
    u64 all_w = 0;
    for (int r = 0; r < blocks; ++r) all_n += get(sh.part_n[0], r), all_w += get(sh.part_w[0], r);
    u64 kept = all_w, unused;
    if (by_k && (unsigned)top_k < all_n) cut = find(false, top_k, by_p, kept);
    if (by_p) {
      const u64 target = (u64)ceil((double)top_p * (double)kept);
      cut = find(true, min(max(target, 1ull), kept), false, unused);
    }
  }

  // ---- the draw
  Pick p = {0.f, 0.f, INT_MAX, INT_MAX};
  const float* e = s.d_noise + b * s.noise_stride + lo;
  for (int i = tid; i < n; i += kThreads) {
    const float x = value(vals[i]);
    if (x == row.m) p.first = min(p.first, lo + i);
    if (row.first || !(x > -INFINITY) || (cut && order_of(x, lo + i) < cut)) continue;
    const float w = row.weight(x);
    if (min_p > 0.f && !(w >= min_p)) continue;
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e[i]));
    const float score = w * r;
    if (score > p.score && score < INFINITY) p.score = score, p.logit = x, p.id = lo + i;
  }
  p = best_warp(p);
  if (lane == 0) sh.picks[warp] = p;
  __syncthreads();
  if (warp == 0) {
    p = best_warp(sh.picks[lane % kWarps]);
    if (lane == 0) {
      put(sh.pick[rank].score, p.score, 0);
      put(sh.pick[rank].logit, p.logit, 0);
      put(sh.pick[rank].id, p.id, 0);
      put(sh.pick[rank].first, p.first, 0);
    }
  }
  cluster_sync();
  if (rank == 0 && warp == 0) {
    p = best_warp(sh.pick[lane % blocks]);
    z = sum_warp(lane < blocks ? sh.zs[lane] : 0.f);
    if (lane == 0) {
      const bool drawn = p.score > 0.f;
      const int token = drawn ? p.id : p.first;
      const float x = drawn ? p.logit : row.m;
      s.d_tokens[b] = token;
      if (s.d_logprob) s.d_logprob[b] = fminf((-row.below(x) * row.c2 - log2f(z)) * kLn2, 0.f);
      s.d_status[b] = token == s.eos ? GRID_ST_COMPLETE : GRID_ST_OK;
    }
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
  SampleArgs a = {*s, 1, 0};
  while (a.blocks < kMaxBlocks && s->V > 4096 * a.blocks) a.blocks *= 2;
  a.each = ((s->V + a.blocks - 1) / a.blocks + 31) & ~31;
  const size_t smem = kSharedRoom + 2 * (size_t)(kBins / a.blocks) * 12 + (size_t)a.each * size;
  auto go = [&](auto kernel, std::atomic<uint64_t>& ready) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    // (the room for shared memory is set once per device)
    if (e == cudaSuccess && !(dev < 64 && ready.load() >> dev & 1)) {
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 << 10);
      if (e == cudaSuccess && dev < 64) ready.fetch_or(1ull << dev);
    }
    if (e != cudaSuccess) return e;
    return launch_cluster(kernel, dim3((unsigned)(s->B * a.blocks)), dim3(kThreads), smem, a.blocks, (cudaStream_t)stream, a);
  };
  static std::atomic<uint64_t> ready[2];
  if (size == 4)
    GRID_CUDA(go(k_sample<float>, ready[0]));
  else
    GRID_CUDA(go(k_sample<uint16_t>, ready[1]));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}
