// Verification of drafted tokens against the masked target distribution, from
// given random numbers (grid_draft_verify).
//
// For row b and position k let l be the logits, A the admitted ids, c = 1/T,
// m = max_A l and s = sum_A exp((l - m) c), so that p(i) = exp((l_i - m) c) / s.
// k_stats computes (m, s, first largest id) of pieces of every position's
// logits in one pass: per thread a running maximum, the sum rescaled when it
// grows; pieces are joined by the same rule.  k_draw joins the pieces of its
// row, walks the acceptance tests u q(x) < p(x) to the first refusal n, and
// draws the next token from position n alone: argmax w_i / e_i needs no running
// sum over the vocabulary, so the order of the additions decides no token.
//
// Both kernels are bound by the bytes they read; each id's mask bit is looked
// at first, and 16 bytes of logits that hold no admitted id are not read.
#include <cfloat>
#include <cmath>

#include "grid_state.cuh"

namespace grid {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxPieces = 64;  // of one position's logits
constexpr int kMaxDraft = 64;
constexpr int kBlocksPerSm = 8;
constexpr float kLog2e = 1.4426950408889634f;

// Exponent and base are fp32: arguments are differences to the maximum, so
// the product with c log2 e is off by 2^-24 of its size.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct Stat {
  float m, s;  // largest admitted logit (-inf: none), sum of exp((l - m) c)
  int id;      // first id that has it
};

__device__ __forceinline__ Stat join(const Stat& a, const Stat& b, float c2) {
  Stat r;
  r.m = fmaxf(a.m, b.m);
  const float z = r.m > -INFINITY ? r.m : 0.f;
  r.s = a.s * exp2_fast((a.m - z) * c2) + b.s * exp2_fast((b.m - z) * c2);
  r.id = a.m == b.m ? min(a.id, b.id) : a.m > b.m ? a.id : b.id;
  return r;
}

__device__ __forceinline__ Stat join_warp(Stat x, float c2) {
  for (int o = 16; o; o >>= 1) {
    Stat y;
    y.m = __shfl_xor_sync(~0u, x.m, o);
    y.s = __shfl_xor_sync(~0u, x.s, o);
    y.id = __shfl_xor_sync(~0u, x.id, o);
    x = join(x, y, c2);
  }
  return x;
}

// NaN counts as -inf, +inf as the largest finite value.
__device__ __forceinline__ float clean(float l) { return fminf(fmaxf(l, -INFINITY), FLT_MAX); }
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }  // bf16

// The row's 1/T (1 for a greedy row) and whether it is greedy.
__device__ __forceinline__ float inv_temp(const grid_draft_step& a, int b, bool& greedy) {
  const float t = a.d_temperature ? a.d_temperature[b] : 1.f;
  greedy = !(t > 0.f);
  return greedy ? 1.f : fminf(1.f / t, FLT_MAX);
}
__device__ __forceinline__ float scale2(float inv) { return fminf(inv * kLog2e, FLT_MAX); }
__device__ __forceinline__ int draft_len(const grid_draft_step& a, int b) {
  return a.d_draft_len ? min(max(a.d_draft_len[b], 0), a.K) : a.K;
}

// Mask bits of ids t .. t + n - 1, the lowest bit first (n <= 32; bits past them are undefined).
__device__ __forceinline__ uint32_t mask_bits(const uint32_t* mask, int W, int t, int n) {
  if (!mask) return ~0u;
  const int w = t >> 5, sh = t & 31;
  const uint32_t lo = mask[w];
  const uint32_t hi = sh + n > 32 && w + 1 < W ? mask[w + 1] : 0u;
  return __funnelshift_r(lo, hi, sh);
}

template <typename T>
__device__ __forceinline__ const T* logits_at(const grid_draft_step& a, int b, int k) {
  return static_cast<const T*>(a.d_logits) + b * a.logit_stride[0] + k * a.logit_stride[1];
}
__device__ __forceinline__ const uint32_t* mask_at(const grid_draft_step& a, int b, int k) {
  return a.d_mask ? a.d_mask + b * a.mask_stride[0] + k * a.mask_stride[1] : nullptr;
}

__device__ __forceinline__ void take(Stat& x, float l, int id, float c2) {
  if (l > x.m) {
    x.s *= exp2_fast((x.m - l) * c2);
    x.m = l;
    x.id = id;
  }
  if (l > -INFINITY) x.s += exp2_fast((l - x.m) * c2);
}

// One piece of one position: block (position row) * pieces + piece.  Pieces
// are cut where the position's 16-byte lines begin, so that rows of any
// alignment are read in whole lines; the ids before the first line belong to
// piece 0, those after the last to the last piece.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_stats(const grid_draft_step a, Stat* __restrict__ stats, int pieces,
                                                    int piece) {
  constexpr int kVec = 16 / sizeof(T), kUnroll = 4;
  const int row = blockIdx.x / pieces, pc = blockIdx.x - row * pieces;
  const int b = row / (a.K + 1), k = row - b * (a.K + 1);
  pdl_wait();
  if (k > draft_len(a, b)) return;
  bool greedy;
  const float c2 = scale2(inv_temp(a, b, greedy));
  const T* l = logits_at<T>(a, b, k);
  const uint32_t* mask = mask_at(a, b, k);
  const int W = (a.V + 31) >> 5, tid = threadIdx.x;
  const int head = min(a.V, (int)((16 - ((uintptr_t)l & 15)) & 15) / (int)sizeof(T));
  const long long from = (long long)head + (long long)pc * piece;
  const int lo = (int)min((long long)a.V, from), hi = (int)min((long long)a.V, from + piece);
  Stat x{-INFINITY, 0.f, INT_MAX};
  if (pc == 0 && tid < head && (mask_bits(mask, W, tid, 1) & 1)) take(x, clean(value(l[tid])), tid, c2);
  const int lines = (hi - lo) / kVec;
  for (int v = tid; v < lines; v += kThreads * kUnroll) {
    uint32_t bits[kUnroll];
    uint4 raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int at = v + u * kThreads;
      bits[u] = at < lines ? mask_bits(mask, W, lo + at * kVec, kVec) & ((1u << kVec) - 1) : 0u;
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      raw[u] = make_uint4(0, 0, 0, 0);
      if (bits[u]) raw[u] = __ldcs(reinterpret_cast<const uint4*>(l + lo + (v + u * kThreads) * kVec));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (!bits[u]) continue;
      const uint32_t r[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
      float y[kVec], top = -INFINITY;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        float f;
        if constexpr (sizeof(T) == 4)
          f = __uint_as_float(r[e]);
        else
          f = __uint_as_float(e & 1 ? r[e / 2] & 0xFFFF0000u : r[e / 2] << 16);
        y[e] = (bits[u] >> e) & 1 ? clean(f) : -INFINITY;
        top = fmaxf(top, y[e]);
      }
      if (top > x.m) {
        x.s *= exp2_fast((x.m - top) * c2);
        x.m = top;
#pragma unroll
        for (int e = kVec - 1; e >= 0; --e)
          if (y[e] == top) x.id = lo + (v + u * kThreads) * kVec + e;
      }
      if (x.m > -INFINITY) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) x.s += exp2_fast((y[e] - x.m) * c2);
      }
    }
  }
  // (the last piece's ids past the last whole line)
  const int t = lo + lines * kVec + tid;
  if (t < hi && (mask_bits(mask, W, t, 1) & 1)) take(x, clean(value(l[t])), t, c2);
  __shared__ Stat sh[kWarps];
  x = join_warp(x, c2);
  if ((tid & 31) == 0) sh[tid >> 5] = x;
  __syncthreads();
  if (tid < 32) {
    x = tid < kWarps ? sh[tid] : Stat{-INFINITY, 0.f, INT_MAX};
    x = join_warp(x, c2);
    if (tid == 0) stats[(size_t)row * pieces + pc] = x;
  }
}

// Best score so far and the first id that has it, for the residual weights
// and for the target's own.
struct Best {
  float r, p;
  int rid, pid;
};
__device__ __forceinline__ void better(float& s, int& id, float t, int j) {
  if (t > s || (t == s && j < id)) {
    s = t;
    id = j;
  }
}
__device__ __forceinline__ Best best_warp(Best x) {
  for (int o = 16; o; o >>= 1) {
    const Best y{__shfl_xor_sync(~0u, x.r, o), __shfl_xor_sync(~0u, x.p, o), __shfl_xor_sync(~0u, x.rid, o),
                 __shfl_xor_sync(~0u, x.pid, o)};
    better(x.r, x.rid, y.r, y.rid);
    better(x.p, x.pid, y.p, y.pid);
  }
  return x;
}

// The draw of one row: block row * parts + part scores its part of the
// vocabulary at the row's position n; the last of the row's blocks writes the
// outcome.  Every block of a row finds n by itself, from the same numbers.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_draw(const grid_draft_step a, const Stat* __restrict__ stats, int pieces,
                                                   Best* __restrict__ best, int* __restrict__ done, int parts,
                                                   int part) {
  constexpr int kUnroll = 4;
  const int b = blockIdx.x / parts, pt = blockIdx.x - b * parts;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __shared__ Stat at[kMaxDraft + 1];
  __shared__ float lx[kMaxDraft];  // logits of the drafted ids
  __shared__ int ok[kMaxDraft + 1];
  __shared__ Best sh[kWarps];
  __shared__ int last;
  pdl_wait();
  bool greedy;
  const float inv = inv_temp(a, b, greedy), c2 = scale2(inv);
  const int nd = draft_len(a, b);
  for (int k = warp; k <= nd; k += kWarps) {
    const Stat* src = stats + ((size_t)b * (a.K + 1) + k) * pieces;
    Stat x{-INFINITY, 0.f, INT_MAX};
    for (int i = lane; i < pieces; i += 32) x = join(x, src[i], c2);
    x = join_warp(x, c2);
    if (lane == 0) {
      at[k] = x;
      ok[k] = 0;
      if (k < nd) {
        const int id = a.d_draft[(size_t)b * a.K + k];
        const uint32_t* mask = mask_at(a, b, k);
        float l = -INFINITY;
        if (id >= 0 && id < a.V && (!mask || (mask[id >> 5] >> (id & 31) & 1)))
          l = clean(value(logits_at<T>(a, b, k)[id]));
        lx[k] = l;
        if (l > -INFINITY) {
          const float q = a.d_probs ? a.d_probs[b * a.prob_stride[0] + k * a.prob_stride[1] + id] : 1.f;
          const float p = exp2_fast((l - x.m) * c2) / x.s;
          ok[k] = greedy ? id == x.id : a.d_u[(size_t)b * a.K + k] * q < p;
          if (ok[k] && id == a.eos) ok[k] = 2;
        }
      }
    }
  }
  __syncthreads();
  int n = 0;
  bool ended = false;
  while (n < nd && ok[n] && !ended) ended = ok[n++] == 2;
  const Stat x = at[min(n, nd)];
  const bool empty = !ended && !(x.m > -INFINITY);
  const bool drawn = !ended && !empty;
  Best z{0.f, 0.f, INT_MAX, INT_MAX};
  if (drawn && !greedy) {
    const T* l = logits_at<T>(a, b, n);
    const uint32_t* mask = mask_at(a, b, n);
    const bool refused = n < nd;
    const float* q = refused && a.d_probs ? a.d_probs + b * a.prob_stride[0] + n * a.prob_stride[1] : nullptr;
    const int out = refused && !q ? a.d_draft[(size_t)b * a.K + n] : -1;
    const float* e = a.d_noise + b * a.noise_stride;
    const int hi = (int)min((long long)a.V, (long long)(pt + 1) * part);
    for (int i = pt * part + tid; i < hi; i += kThreads * kUnroll) {
      float lv[kUnroll], ev[kUnroll], qv[kUnroll];
      bool in[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int j = i + u * kThreads;
        in[u] = j < hi && (!mask || (mask[j >> 5] >> (j & 31) & 1));
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int j = i + u * kThreads;
        lv[u] = in[u] ? value(l[j]) : 0.f;
        ev[u] = in[u] ? e[j] : 0.f;
        qv[u] = in[u] && q ? q[j] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int j = i + u * kThreads;
        if (!in[u] || !(ev[u] > 0.f)) continue;
        const float p = exp2_fast((clean(lv[u]) - x.m) * c2) / x.s;
        const float r = j == out ? 0.f : fmaxf(p - qv[u], 0.f);
        const float sr = r / ev[u];
        if (sr > z.r) z.r = sr, z.rid = j;
        if (refused) {
          const float sp = p / ev[u];
          if (sp > z.p) z.p = sp, z.pid = j;
        }
      }
    }
    z = best_warp(z);
    if (lane == 0) sh[warp] = z;
    __syncthreads();
    if (warp == 0) {
      z = best_warp(lane < kWarps ? sh[lane] : Best{0.f, 0.f, INT_MAX, INT_MAX});
      if (lane == 0) {
        if (parts > 1) {
          best[(size_t)b * parts + pt] = z;
          __threadfence();
          last = atomicAdd(&done[b], 1) == parts - 1;
          __threadfence();
        } else {
          sh[0] = z;
          last = 1;
        }
      }
    }
    __syncthreads();
    if (!last) return;
    if (parts > 1 && warp == 0) {
      z = Best{0.f, 0.f, INT_MAX, INT_MAX};
      for (int i = lane; i < parts; i += 32) {
        const Best* y = best + (size_t)b * parts + i;
        better(z.r, z.rid, __ldcg(&y->r), __ldcg(&y->rid));
        better(z.p, z.pid, __ldcg(&y->p), __ldcg(&y->pid));
      }
      z = best_warp(z);
      if (lane == 0) {
        sh[0] = z;
        done[b] = 0;
      }
    }
    __syncthreads();
    z = sh[0];
  } else if (pt) {
    return;
  }
  const int token = !drawn ? -1 : greedy ? x.id : z.r > 0.f ? z.rid : z.p > 0.f ? z.pid : x.id;
  for (int k = tid; k <= a.K; k += kThreads) {
    const int id = k < n ? a.d_draft[(size_t)b * a.K + k] : k == n ? token : -1;
    a.d_tokens[(size_t)b * (a.K + 1) + k] = id;
    if (a.d_logprob) {
      float v = 0.f;
      if (id >= 0) {
        const float l = k < n ? lx[k] : clean(value(logits_at<T>(a, b, k)[id]));
        v = (l - at[k].m) * inv - logf(at[k].s);
      }
      a.d_logprob[(size_t)b * (a.K + 1) + k] = v;
    }
  }
  if (tid == 0) {
    a.d_accepted[b] = n;
    a.d_status[b] = ended || (drawn && token == a.eos) ? GRID_ST_COMPLETE : empty ? GRID_ST_EMPTY_MASK : GRID_ST_OK;
  }
}

}  // namespace
}  // namespace grid

using namespace grid;

struct grid_drafts {
  int B = 0, K = 0, V = 0, sms = 152;
  Stat* stats = nullptr;
  Best* best = nullptr;
  int* done = nullptr;
  Arena mem;
};

extern "C" int grid_drafts_create(int32_t B, int32_t K, int32_t V, grid_drafts** out) {
  if (!out || B <= 0 || K < 0 || K > kMaxDraft || V <= 0)
    return set_error(GRID_E_INVALID_ARG, "grid_drafts_create: B and V are positive, K in 0 .. 64");
  if (B > 65535) return set_error(GRID_E_TOO_LARGE, "grid_drafts_create: more than 65535 rows");
  grid_drafts* d = new grid_drafts;
  d->B = B;
  d->K = K;
  d->V = V;
  int rc = GRID_OK, dev = 0;
  cudaError_t e = cudaSuccess;
  // (a call cuts n positions, or rows, into at most n + kBlocksPerSm * sms pieces)
  if ((e = cudaGetDevice(&dev)) == cudaSuccess &&
      (e = cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, dev)) == cudaSuccess &&
      !(rc = d->mem.alloc(((size_t)B * (K + 1) + kBlocksPerSm * d->sms) * sizeof(Stat), (void**)&d->stats)) &&
      !(rc = d->mem.alloc(((size_t)B + kBlocksPerSm * d->sms) * sizeof(Best), (void**)&d->best)) &&
      !(rc = d->mem.alloc((size_t)B * sizeof(int), (void**)&d->done)) &&
      (e = cudaMemset(d->done, 0, (size_t)B * sizeof(int))) == cudaSuccess)
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
  cudaStream_t st = (cudaStream_t)stream;
  // Pieces of a position and parts of a draw: as many blocks as keep every SM
  // busy, and no block of fewer than 2,048 ids.
  auto cut = [&](long long rows, int& count, int& size_) {
    const long long want = ((long long)kBlocksPerSm * d->sms + rows - 1) / rows;
    const int most = std::min(kMaxPieces, (s->V + 2047) / 2048);
    count = (int)std::max(1LL, std::min<long long>(want, most));
    size_ = ((s->V + count - 1) / count + 31) & ~31;
    count = (s->V + size_ - 1) / size_;
  };
  int pieces, piece, parts, part;
  const long long rows = (long long)s->B * (s->K + 1);
  cut(rows, pieces, piece);
  cut(s->B, parts, part);
  auto go = [&](auto stats, auto draw) {
    cudaError_t e = launch_pdl(stats, dim3((unsigned)(rows * pieces)), dim3(kThreads), 0, st, *s, d->stats, pieces, piece);
    if (e != cudaSuccess) return e;
    return launch_pdl(draw, dim3((unsigned)(s->B * parts)), dim3(kThreads), 0, st, *s, (const Stat*)d->stats, pieces,
                      d->best, d->done, parts, part);
  };
  GRID_CUDA(size == 4 ? go(k_stats<float>, k_draw<float>) : go(k_stats<uint16_t>, k_draw<uint16_t>));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}
