// A chunk of tokens through a model's attention: the paged cache's append
// (grid_kv_append) and the attention over it (grid_kv_attend).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "grid_state.cuh"

namespace grid {
namespace {

struct Chunk {  // grid_kv_chunk with the cache's geometry
  const int32_t* table;
  const int32_t* len;
  const int32_t* start;
  long long table_stride;
  int max_pages, B, N, n_pages, log_page, T;  // T: tokens of every row where start is NULL
};

// Row b's tokens [a, a + n) and its first position; false where they are not in order.
__device__ __forceinline__ bool row_span(const Chunk& c, int b, int& a, int& n, int& len) {
  a = c.start ? c.start[b] : b * c.T;
  const int z = c.start ? c.start[b + 1] : a + c.T;
  len = c.len[b];
  n = z - a;
  return a >= 0 && z >= a && z <= c.N && len >= 0 && (long long)len + n <= (long long)c.max_pages << c.log_page;
}

// The row of token i, or -1: the last b with start[b] <= i, by a warp (each
// step looks at 32 entries at once; at most four steps for 65,535 rows).
__device__ __forceinline__ int row_of(const Chunk& c, int i, int lane) {
  if (!c.start) return i / c.T;
  int lo = 0, n = c.B + 1;  // start[lo] <= i is known once found, the answer lies in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int at = lo + lane * step;
    const unsigned in = __ballot_sync(~0u, lane * step < n && c.start[min(at, c.B)] <= i);
    if (!in) return -1;
    const int k = 31 - __clz(in);
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo < c.B && c.start[lo] <= i && i < c.start[lo + 1] ? lo : -1;
}

// Page of position p of row b, or -1 when its id is outside the cache.
__device__ __forceinline__ int page_of(const Chunk& c, int b, int p) {
  const int id = c.table[b * c.table_stride + (p >> c.log_page)];
  return id >= 0 && id < c.n_pages ? id : -1;
}

__device__ __forceinline__ float lo_of(uint32_t w, __nv_bfloat16) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_of(uint32_t w, __nv_bfloat16) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float lo_of(uint32_t w, __half) { return __half2float(__ushort_as_half((uint16_t)w)); }
__device__ __forceinline__ float hi_of(uint32_t w, __half) { return __half2float(__ushort_as_half((uint16_t)(w >> 16))); }
__device__ __forceinline__ uint32_t pack_of(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_of(float a, float b, __half) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ void unpack8(const uint4& r, float* x) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = lo_of(w[i], T());
    x[2 * i + 1] = hi_of(w[i], T());
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(pack_of(x[0], x[1], T()), pack_of(x[2], x[3], T()), pack_of(x[4], x[5], T()), pack_of(x[6], x[7], T()));
}

// ---------------------------------------------------------------------------
// Append.  A head vector is D / 8 lanes of 16 bytes, so a warp holds 512 / (2 D)
// heads at once and kUnroll such groups of one token; the rotation's partner
// values come by shuffle.  Bound by the bytes moved.
struct AppendArgs {
  Chunk c;
  const void *q, *k, *v, *qw, *kw;
  void *qo, *kp, *vp;
  long long qs[2], ks[2], vs[2], qos[2], kps[3], vps[3];
  const float *cos, *sin;
  float eps;
  int H, Hk, rot, pairs, n_pos, groups;  // groups: of heads per token
  int32_t* status;
};

constexpr int kAppendUnroll = 4, kAppendWarps = 4;

template <typename T, int D>
__global__ void __launch_bounds__(kAppendWarps * 32) k_append(const AppendArgs a, int token_blocks) {
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes;  // lanes of a head, heads of a warp's load
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  const Chunk& c = a.c;
  if ((int)blockIdx.x >= token_blocks) {  // a warp per row: its status
    const int b = ((int)blockIdx.x - token_blocks) * kAppendWarps + warp;
    if (b >= c.B) return;
    int s, n, len;
    bool ok = row_span(c, b, s, n, len) && (!a.cos || n == 0 || len + n <= a.n_pos);
    if (ok && n)
      for (int p = (len >> c.log_page) + lane; p <= (len + n - 1) >> c.log_page; p += 32)
        ok = ok && page_of(c, b, p << c.log_page) >= 0;
    ok = __all_sync(~0u, ok);
    if (lane == 0) a.status[b] = ok ? GRID_ST_OK : GRID_ST_PAGES;
    return;
  }
  const long long item = (long long)blockIdx.x * kAppendWarps + warp;
  const int i = (int)(item / a.groups), group = (int)(item - (long long)i * a.groups);
  if (i >= c.N) return;
  const int nq = a.q ? a.H : 0, heads = nq + 2 * a.Hk;
  const int l = lane % kLanes, e = l * 8;
  uint4 raw[kAppendUnroll];
  int head[kAppendUnroll];
#pragma unroll
  for (int u = 0; u < kAppendUnroll; ++u) {
    const int h = (group * kAppendUnroll + u) * kHeads + lane / kLanes;
    head[u] = h;
    raw[u] = make_uint4(0, 0, 0, 0);
    if (h >= heads) continue;
    const T* src = h < nq ? (const T*)a.q + i * a.qs[0] + h * a.qs[1]
                   : h < nq + a.Hk ? (const T*)a.k + i * a.ks[0] + (h - nq) * a.ks[1]
                                   : (const T*)a.v + i * a.vs[0] + (h - nq - a.Hk) * a.vs[1];
    raw[u] = __ldcs(reinterpret_cast<const uint4*>(src + e));
  }
  const int b = row_of(c, i, lane);
  if (b < 0) return;
  int s, n, len;
  if (!row_span(c, b, s, n, len)) return;
  const int pos = len + i - s;
  if (a.cos && pos >= a.n_pos) return;
  const int page = page_of(c, b, pos);
  if (page < 0) return;
  const int off = pos & ((1 << c.log_page) - 1);
  // cosines and sines of this lane's values, -sin where the value is the first of its pair
  float cs[8], sn[8];
  const bool turned = a.cos && e < a.rot;
#pragma unroll
  for (int j = 0; j < 8; ++j) cs[j] = 1.f, sn[j] = 0.f;
  const int half = a.rot / 2;
  if (turned) {
    const float* ct = a.cos + (long long)pos * half;
    const float* st = a.sin + (long long)pos * half;
    if (a.pairs) {
      const float4 x = *reinterpret_cast<const float4*>(ct + e / 2), y = *reinterpret_cast<const float4*>(st + e / 2);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        cs[2 * j] = cs[2 * j + 1] = xs[j];
        sn[2 * j] = -ys[j];
        sn[2 * j + 1] = ys[j];
      }
    } else {
      const int m = e < half ? e : e - half;
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        const float4 x = *reinterpret_cast<const float4*>(ct + m + j), y = *reinterpret_cast<const float4*>(st + m + j);
        const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          cs[j + t] = xs[t];
          sn[j + t] = e < half ? -ys[t] : ys[t];
        }
      }
    }
  }
  const int from = turned && !a.pairs ? lane + (e < half ? half / 8 : -(half / 8)) : lane;  // the partner's lane
#pragma unroll
  for (int u = 0; u < kAppendUnroll; ++u) {
    const int h = head[u];
    const bool is_v = h >= nq + a.Hk;
    float x[8];
    unpack8<T>(raw[u], x);
    const void* w = h < nq ? a.qw : a.kw;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += x[j] * x[j];
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (w && !is_v) {
      const float r = 1.f / sqrtf(sum / D + a.eps);
      float g[8];
      unpack8<T>(*reinterpret_cast<const uint4*>((const T*)w + e), g);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = x[j] * r * g[j];
    }
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = a.pairs ? x[j ^ 1] : __shfl_sync(~0u, x[j], from);
    if (h < nq + 2 * a.Hk) {
      if (!is_v && turned) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * cs[j] + y[j] * sn[j];
      }
      T* dst = h < nq ? (T*)a.qo + i * a.qos[0] + h * a.qos[1]
               : !is_v ? (T*)a.kp + page * a.kps[0] + off * a.kps[1] + (h - nq) * a.kps[2]
                       : (T*)a.vp + page * a.vps[0] + off * a.vps[1] + (h - nq - a.Hk) * a.vps[2];
      *reinterpret_cast<uint4*>(dst + e) = is_v ? raw[u] : pack8<T>(x);
    }
  }
}

// ---------------------------------------------------------------------------
// Attention: a warp per token and query head, one key after the other.
struct AttendArgs {
  Chunk c;
  const void *q, *kp, *vp;
  void* out;
  float* lse;
  long long qs[2], os[2], kps[3], vps[3];
  int H, Hk;
  float scale;
  int32_t* status;
};

template <typename T, int D>
__global__ void __launch_bounds__(128) k_attend(const AttendArgs a, int token_blocks) {
  constexpr int kPer = D / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Chunk& c = a.c;
  pdl_wait();
  auto row_ok = [&](int b, int n, int len) {
    bool ok = true;
    if (n)
      for (int p = lane; p <= (len + n - 1) >> c.log_page; p += 32) ok = ok && page_of(c, b, p << c.log_page) >= 0;
    return __all_sync(~0u, ok);
  };
  int s, n, len;
  if ((int)blockIdx.x >= token_blocks) {
    const int b = ((int)blockIdx.x - token_blocks) * 4 + warp;
    if (b >= c.B) return;
    const bool ok = row_span(c, b, s, n, len) && row_ok(b, n, len);
    if (lane == 0) a.status[b] = ok ? GRID_ST_OK : GRID_ST_PAGES;
    return;
  }
  const long long item = (long long)blockIdx.x * 4 + warp;
  const int i = (int)(item / a.H), h = (int)(item - (long long)i * a.H);
  if (i >= c.N) return;
  const int b = row_of(c, i, lane);
  if (b < 0) return;
  const bool ok = row_span(c, b, s, n, len) && row_ok(b, n, len);
  const T* q = (const T*)a.q + i * a.qs[0] + h * a.qs[1];
  float qv[kPer], acc[kPer], m = -INFINITY, z = 0.f;
  for (int j = 0; j < kPer; ++j) {
    qv[j] = (float)q[lane * kPer + j];
    acc[j] = 0.f;
  }
  const int hk = h / (a.H / a.Hk), last = ok ? len + i - s : -1;
  for (int p = 0; p <= last; ++p) {
    const long long page = page_of(c, b, p), off = p & ((1 << c.log_page) - 1);
    const T* k = (const T*)a.kp + page * a.kps[0] + off * a.kps[1] + hk * a.kps[2];
    const T* v = (const T*)a.vp + page * a.vps[0] + off * a.vps[1] + hk * a.vps[2];
    float x = 0.f;
    for (int j = 0; j < kPer; ++j) x += qv[j] * (float)k[lane * kPer + j];
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    x *= a.scale;
    const float top = fmaxf(m, x), f = expf(m - top), w = expf(x - top);
    z = z * f + w;
    for (int j = 0; j < kPer; ++j) acc[j] = acc[j] * f + w * (float)v[lane * kPer + j];
    m = top;
  }
  T* o = (T*)a.out + i * a.os[0] + h * a.os[1];
  for (int j = 0; j < kPer; ++j) o[lane * kPer + j] = (T)(z > 0.f ? acc[j] / z : 0.f);
  if (a.lse && lane == 0) a.lse[(long long)i * a.H + h] = z > 0.f ? m + logf(z) : -INFINITY;
}

bool heads_ok(const grid_heads* h) {
  return h && h->d && (uintptr_t)h->d % 16 == 0 && h->token_stride >= 0 && h->head_stride >= 0 &&
         h->token_stride % 8 == 0 && h->head_stride % 8 == 0;
}

}  // namespace
}  // namespace grid

using namespace grid;

struct grid_kv {
  grid_kv_pages p;
  int log_page = 0, sms = 152;
  Arena mem;
};

// The chunk as the kernels take it; false where its arguments are bad.
static bool make_chunk(const grid_kv* kv, const grid_kv_chunk* ch, Chunk& c) {
  if (!ch || !ch->d_table || !ch->d_len || ch->B <= 0 || ch->n_tokens < 0 || ch->max_pages <= 0 ||
      ch->table_stride < ch->max_pages || ((int64_t)ch->max_pages << kv->log_page) > INT32_MAX ||
      (!ch->d_start && ch->n_tokens % ch->B))
    return false;
  c = Chunk{ch->d_table, ch->d_len, ch->d_start, ch->table_stride, ch->max_pages, ch->B, ch->n_tokens,
            kv->p.n_pages, kv->log_page, ch->n_tokens / ch->B};
  return true;
}

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
  grid_kv* kv = new grid_kv;
  kv->p = *p;
  while (1 << kv->log_page < p->page_size) ++kv->log_page;
  *out = kv;
  return GRID_OK;
}

extern "C" void grid_kv_free(grid_kv* kv) {
  if (!kv) return;
  kv->mem.release();
  delete kv;
}

extern "C" int grid_kv_append(const grid_kv* kv, const grid_kv_chunk* chunk, const grid_heads* k, const grid_heads* v,
                              const grid_heads* q, const grid_heads* q_out, const grid_rotation* rot,
                              const grid_head_norm* norm, int32_t* d_status, void* stream) {
  AppendArgs a = {};
  if (!kv || !d_status || !make_chunk(kv, chunk, a.c) || (chunk->n_tokens && (!heads_ok(k) || !heads_ok(v))) ||
      (q != nullptr) != (q_out != nullptr) || (q && chunk->n_tokens && (!heads_ok(q) || !heads_ok(q_out))))
    return set_error(GRID_E_INVALID_ARG, "grid_kv_append: bad arguments");
  if (rot && (!rot->d_cos || !rot->d_sin || (uintptr_t)rot->d_cos % 16 || (uintptr_t)rot->d_sin % 16 ||
              rot->n_pos <= 0 || rot->rot <= 0 || rot->rot % 16 || rot->rot > kv->p.head_dim))
    return set_error(GRID_E_INVALID_ARG, "grid_kv_append: bad rotation (rot is a multiple of 16 up to head_dim)");
  if (norm && ((uintptr_t)norm->d_q % 16 || (uintptr_t)norm->d_k % 16 || !(norm->eps >= 0.f)))
    return set_error(GRID_E_INVALID_ARG, "grid_kv_append: bad norm");
  if (chunk->B > 65535) return set_error(GRID_E_TOO_LARGE, "grid_kv_append: more than 65535 rows");
  const grid_kv_pages& p = kv->p;
  if (chunk->n_tokens) {
    a.k = k->d, a.v = v->d;
    a.ks[0] = k->token_stride, a.ks[1] = k->head_stride, a.vs[0] = v->token_stride, a.vs[1] = v->head_stride;
    if (q) {
      a.q = q->d, a.qo = q_out->d;
      a.qs[0] = q->token_stride, a.qs[1] = q->head_stride;
      a.qos[0] = q_out->token_stride, a.qos[1] = q_out->head_stride;
    }
  }
  a.kp = p.d_k, a.vp = p.d_v;
  for (int i = 0; i < 3; ++i) a.kps[i] = p.k_stride[i], a.vps[i] = p.v_stride[i];
  if (rot) a.cos = rot->d_cos, a.sin = rot->d_sin, a.rot = rot->rot, a.pairs = rot->pairs, a.n_pos = rot->n_pos;
  if (norm) a.qw = norm->d_q, a.kw = norm->d_k, a.eps = norm->eps;
  a.H = p.n_heads, a.Hk = p.n_kv_heads;
  a.status = d_status;
  const int at_once = kAppendUnroll * (256 / p.head_dim);
  a.groups = ((q ? a.H : 0) + 2 * a.Hk + at_once - 1) / at_once;
  const long long blocks = ((long long)chunk->n_tokens * a.groups + kAppendWarps - 1) / kAppendWarps;
  const int rows = (chunk->B + kAppendWarps - 1) / kAppendWarps;
  if (blocks + rows > INT32_MAX) return set_error(GRID_E_TOO_LARGE, "grid_kv_append: too many head vectors in one call");
  auto go = [&](auto kern) {
    return launch_pdl(kern, dim3((unsigned)(blocks + rows)), dim3(kAppendWarps * 32), 0, (cudaStream_t)stream, a, (int)blocks);
  };
  if (p.dtype == GRID_DTYPE_BF16)
    GRID_CUDA(p.head_dim == 64 ? go(k_append<__nv_bfloat16, 64>) : go(k_append<__nv_bfloat16, 128>));
  else
    GRID_CUDA(p.head_dim == 64 ? go(k_append<__half, 64>) : go(k_append<__half, 128>));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
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
  a.q = query->q.d, a.out = query->out.d, a.lse = query->d_lse;
  a.qs[0] = query->q.token_stride, a.qs[1] = query->q.head_stride;
  a.os[0] = query->out.token_stride, a.os[1] = query->out.head_stride;
  a.kp = p.d_k, a.vp = p.d_v;
  for (int i = 0; i < 3; ++i) a.kps[i] = p.k_stride[i], a.vps[i] = p.v_stride[i];
  a.H = p.n_heads, a.Hk = p.n_kv_heads, a.scale = query->scale, a.status = d_status;
  const long long blocks = ((long long)chunk->n_tokens * a.H + 3) / 4;
  const int rows = (chunk->B + 3) / 4;
  if (blocks + rows > INT32_MAX) return set_error(GRID_E_TOO_LARGE, "grid_kv_attend: too many head vectors in one call");
  auto go = [&](auto kern) {
    return launch_pdl(kern, dim3((unsigned)(blocks + rows)), dim3(128), 0, (cudaStream_t)stream, a, (int)blocks);
  };
  if (p.dtype == GRID_DTYPE_BF16)
    GRID_CUDA(p.head_dim == 64 ? go(k_attend<__nv_bfloat16, 64>) : go(k_attend<__nv_bfloat16, 128>));
  else
    GRID_CUDA(p.head_dim == 64 ? go(k_attend<__half, 64>) : go(k_attend<__half, 128>));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}
