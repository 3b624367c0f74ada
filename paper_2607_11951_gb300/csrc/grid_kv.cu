// The paged cache's append: a chunk's keys and values into their pages, norms
// and rotation on the way (grid_kv_append).
#include <cmath>

#include "grid_kv.cuh"

namespace grid {
namespace {

// A head vector is D / 8 lanes of 16 bytes, so a warp's load holds 512 / (2 D)
// heads; kUnroll of them, all queries, all keys or all values, are a group, and
// a warp takes some groups of one token.  With r = 1 / sqrt(mean(x^2) + eps),
// weights w and the angle's c and s, a value is r (x_i (w_i c) + x_j (w_j s))
// with x_j its partner, which comes by shuffle; the factors in brackets are the
// token's own and made once for all of its heads.
//
// Bound by the bytes moved: the first group is on its way while the token's
// row, length and page are looked up one after the other, each later one while
// the one before is worked on.  A large batch's warps take whole tokens, so that
// the look-ups (3 us) are paid once for 24 KB; a small one's take a group each.
struct AppendArgs {
  Chunk c;
  const void* src[3];       // queries, keys, values
  void* dst[3];             // queries out, the pools of keys and of values
  const void* w[2];         // norm weights of queries and keys
  long long ss[3][2], qos[2], ps[2][3];  // strides of src, of queries out and of the pools
  const float *cos, *sin;
  float eps;
  int H, Hk, rot, pairs, n_pos;
  int groups[3];            // up to the last one of the queries, of the keys, of the values
  int splits;               // warps that a token's groups go to
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
  const int i = (int)(item / a.splits), split = (int)(item - (long long)i * a.splits);
  if (i >= c.N) return;
  const int e = lane % kLanes * 8, mine = lane / kLanes;
  auto kind_of = [&](int group) { return group < a.groups[0] ? 0 : group < a.groups[1] ? 1 : 2; };
  auto head_of = [&](int group, int kind) { return (group - (kind ? a.groups[kind - 1] : 0)) * kAppendUnroll * kHeads + mine; };
  auto fetch = [&](int group, uint4* raw) {
    const int kind = kind_of(group), h = head_of(group, kind), heads = kind ? a.Hk : a.H;
    const T* p = (const T*)a.src[kind] + i * a.ss[kind][0] + h * a.ss[kind][1] + e;
    const long long step = kHeads * a.ss[kind][1];
#pragma unroll
    for (int u = 0; u < kAppendUnroll; ++u)
      if (h + u * kHeads < heads) raw[u] = __ldcs(reinterpret_cast<const uint4*>(p + u * step));
  };
  uint4 ahead[kAppendUnroll] = {};
  fetch(split, ahead);
  const int b = row_of(c, i, lane);
  if (b < 0) return;
  int s, n, len;
  if (!row_span(c, b, s, n, len)) return;
  const int pos = len + i - s;
  if (a.cos && pos >= a.n_pos) return;
  const int page = page_of(c, b, pos);
  if (page < 0) return;
  const int off = pos & ((1 << c.log_page) - 1), half = a.rot / 2;
  const bool turned = a.cos && e < a.rot;
  const int across = turned && !a.pairs ? (e < half ? half : -half) : 0;  // to the partner's value, where it is another lane's
  const int from = lane + across / 8;
  float wc[8], ws[8];  // w_i c and w_j s, s with the sign that it has for this value
  int kind = -1;
#pragma unroll 1
  for (int group = split; group < a.groups[2]; group += a.splits) {
    uint4 raw[kAppendUnroll];
#pragma unroll
    for (int u = 0; u < kAppendUnroll; ++u) raw[u] = ahead[u];
    if (group + a.splits < a.groups[2]) fetch(group + a.splits, ahead);
    const bool changed = kind != kind_of(group);
    kind = kind_of(group);
    const int h = head_of(group, kind), heads = kind ? a.Hk : a.H;
    T* dst = (T*)a.dst[kind] + e;
    dst += kind ? page * a.ps[kind - 1][0] + off * a.ps[kind - 1][1] + h * a.ps[kind - 1][2] : i * a.qos[0] + h * a.qos[1];
    const long long step = kHeads * (kind ? a.ps[kind - 1][2] : a.qos[1]);
    if (kind == 2) {
#pragma unroll
      for (int u = 0; u < kAppendUnroll; ++u)
        if (h + u * kHeads < heads) *reinterpret_cast<uint4*>(dst + u * step) = raw[u];
      continue;
    }
    const T* w = (const T*)a.w[kind];
    if (changed) {
      float wp[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) wc[j] = wp[j] = 1.f, ws[j] = 0.f;
      if (w) {
        unpack8<T>(*reinterpret_cast<const uint4*>(w + e), wc);
        unpack8<T>(*reinterpret_cast<const uint4*>(w + e + across), wp);
      }
      if (turned) {
        const int m = a.pairs ? e / 2 : e < half ? e : e - half;
        const float* ct = a.cos + (long long)pos * half + m;
        const float* st = a.sin + (long long)pos * half + m;
        float cs[8], sn[8];
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          if (a.pairs && j) break;
          const float4 x = *reinterpret_cast<const float4*>(ct + j), y = *reinterpret_cast<const float4*>(st + j);
          cs[j] = x.x, cs[j + 1] = x.y, cs[j + 2] = x.z, cs[j + 3] = x.w;
          sn[j] = y.x, sn[j + 1] = y.y, sn[j + 2] = y.z, sn[j + 3] = y.w;
        }
        float own[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) own[j] = wc[j];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (a.pairs) {
            wc[j] = own[j] * cs[j / 2];
            ws[j] = own[j ^ 1] * (j & 1 ? sn[j / 2] : -sn[j / 2]);
          } else {
            wc[j] = own[j] * cs[j];
            ws[j] = wp[j] * (e < half ? -sn[j] : sn[j]);
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kAppendUnroll; ++u) {
      float x[8], y[8], r = 1.f;
      unpack8<T>(raw[u], x);
      if (w) {
        float sum = x[0] * x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) sum = fmaf(x[j], x[j], sum);
#pragma unroll
        for (int o = kLanes / 2; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        r = rsqrtf(sum * (1.f / D) + a.eps);
      }
      if (a.cos && !a.pairs) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __shfl_sync(~0u, x[j], from);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j ^ 1];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (turned ? fmaf(x[j], wc[j], y[j] * ws[j]) : x[j] * wc[j]) * r;
      if (h + u * kHeads < heads) *reinterpret_cast<uint4*>(dst + u * step) = pack8<T>(x);
    }
  }
}

}  // namespace
}  // namespace grid

using namespace grid;

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
  const int at_once = kAppendUnroll * (256 / p.head_dim);
  auto heads = [&](int kind, const grid_heads* h, int count) {
    if (chunk->n_tokens && h) a.src[kind] = h->d, a.ss[kind][0] = h->token_stride, a.ss[kind][1] = h->head_stride;
    a.groups[kind] = (kind ? a.groups[kind - 1] : 0) + (h ? (count + at_once - 1) / at_once : 0);
  };
  heads(0, q, p.n_heads);
  heads(1, k, p.n_kv_heads);
  heads(2, v, p.n_kv_heads);
  if (q) a.dst[0] = q_out->d, a.qos[0] = q_out->token_stride, a.qos[1] = q_out->head_stride;
  a.dst[1] = p.d_k, a.dst[2] = p.d_v;
  for (int i = 0; i < 3; ++i) a.ps[0][i] = p.k_stride[i], a.ps[1][i] = p.v_stride[i];
  if (rot) a.cos = rot->d_cos, a.sin = rot->d_sin, a.rot = rot->rot, a.pairs = rot->pairs, a.n_pos = rot->n_pos;
  if (norm) a.w[0] = norm->d_q, a.w[1] = norm->d_k, a.eps = norm->eps;
  a.H = p.n_heads, a.Hk = p.n_kv_heads;
  a.status = d_status;
  // (whole tokens where their warps fill the SMs anyway)
  a.splits = std::max(1, std::min(a.groups[2], 32 * kv->sms / std::max(1, chunk->n_tokens)));
  const long long blocks = ((long long)chunk->n_tokens * a.splits + kAppendWarps - 1) / kAppendWarps;
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
