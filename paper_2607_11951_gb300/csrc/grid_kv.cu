// The paged cache's append: a chunk's keys and values into their pages, norms
// and rotation on the way (grid_kv_append).
#include <cmath>

#include "grid_kv.cuh"

namespace grid {
namespace {

// A head vector is D / 8 lanes of 16 bytes, so a warp's load holds 512 / (2 D)
// heads; kUnroll of them are a group, and a warp takes some groups of one
// token.  The rotation's partner values come by shuffle.  Bound by the bytes
// moved: the first group is on its way while the token's row, length and page
// are looked up one after the other, each later one while the one before is
// worked on.  A large batch's warps take whole tokens, so that the look-ups
// (3 us) are paid once for 24 KB; a small one's take a group each.
struct AppendArgs {
  Chunk c;
  const void *q, *k, *v, *qw, *kw;
  void *qo, *kp, *vp;
  long long qs[2], ks[2], vs[2], qos[2], kps[3], vps[3];
  const float *cos, *sin;
  float eps;
  int H, Hk, rot, pairs, n_pos;
  int groups, splits;  // groups of heads per token, warps that they go to
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
  const int nq = a.q ? a.H : 0, heads = nq + 2 * a.Hk;
  const int l = lane % kLanes, e = l * 8;
  auto fetch = [&](int group, uint4* raw) {
#pragma unroll
    for (int u = 0; u < kAppendUnroll; ++u) {
      const int h = (group * kAppendUnroll + u) * kHeads + lane / kLanes;
      const T* src = h < nq ? (const T*)a.q + i * a.qs[0] + h * a.qs[1]
                     : h < nq + a.Hk ? (const T*)a.k + i * a.ks[0] + (h - nq) * a.ks[1]
                                     : (const T*)a.v + i * a.vs[0] + (h - nq - a.Hk) * a.vs[1];
      raw[u] = make_uint4(0, 0, 0, 0);
      if (h < heads) raw[u] = __ldcs(reinterpret_cast<const uint4*>(src + e));
    }
  };
  uint4 ahead[kAppendUnroll];
  fetch(split, ahead);
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
#pragma unroll 1
  for (int group = split; group < a.groups; group += a.splits) {
    uint4 raw[kAppendUnroll];
#pragma unroll
    for (int u = 0; u < kAppendUnroll; ++u) raw[u] = ahead[u];
    if (group + a.splits < a.groups) fetch(group + a.splits, ahead);
#pragma unroll
    for (int u = 0; u < kAppendUnroll; ++u) {
      const int h = (group * kAppendUnroll + u) * kHeads + lane / kLanes;
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
  // (whole tokens where their warps fill the SMs anyway)
  a.splits = std::max(1, std::min(a.groups, 32 * kv->sms / std::max(1, chunk->n_tokens)));
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
