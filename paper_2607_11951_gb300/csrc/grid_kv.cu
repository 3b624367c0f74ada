// The paged cache's append: a chunk's keys and values into their pages, norms
// and rotation on the way (grid_kv_append).
#include <cmath>

#include "grid_kv.cuh"

namespace grid {
namespace {

// A head vector is D / 8 lanes of 8 values, so a warp's load holds 256 / D
// heads; eight heads, all queries, all keys or all values, are a group, and a
// warp takes some groups of one token.  With r = 1 / sqrt(mean(x^2) + eps),
// weights w and the angle's c and s, a value is r (x_i (w_i c) + x_j (w_j s))
// with x_j its partner, in fp32, rounded once to the cache's type; the factors
// in brackets are the token's own and made once for all of its heads.  A lane's
// values are two times four neighbours, one in each half of what is turned, so
// that partners are one lane's and its arithmetic is on two values at once.
//
// Bound by the bytes moved: 32 prompts of 2,000 tokens (32 + 8 heads of 128,
// normed and turned, 1.19 GB) take 187 us, 6.4 TB/s (partners by shuffle: 221
// us, with 61% of the issue slots taken).  The first group is on its way while
// the token's row, length and page are looked up one after the other, each later
// one while the one before is worked on.  A large batch's warps take whole
// tokens, so that the look-ups (3 us) are paid once for 24 KB; a small one's take
// a group each (256 tokens 3.3 us, one 2.2).  Eight heads at once: four took 197
// us, and twelve 203.
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
  const int32_t* depth;     // of the tokens in their trees, or NULL: their order in the row
  int32_t* status;
};

constexpr int kGroup = 8, kAppendWarps = 4;

template <typename T, int D>
__global__ void __launch_bounds__(kAppendWarps * 32, D == 128 ? 6 : 8) k_append(const AppendArgs a, int token_blocks) {
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes, kUnroll = kGroup / kHeads;  // lanes of a head, heads of a load, loads
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_next();
  const Chunk& c = a.c;
  if ((int)blockIdx.x >= token_blocks) {  // a warp per row: its status
    const int b = ((int)blockIdx.x - token_blocks) * kAppendWarps + warp;
    if (b >= c.B) return;
    int s, n, len;
    bool ok = row_span(c, b, s, n, len) && (!a.cos || a.depth || n == 0 || len + n <= a.n_pos);
    if (ok && a.cos && a.depth)
      for (int i = lane; i < n; i += 32) ok = ok && a.depth[s + i] >= 0 && a.depth[s + i] < a.n_pos - len;
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
  // values at[0] .. +3 and at[1] .. +3 of a head, the pairs' angles from `angle` on
  const int place = lane % kLanes, mine = lane / kLanes, half = a.rot / 2;
  const bool turned = place * 8 < a.rot, halves = turned && !a.pairs;
  const int at[2] = {halves ? place * 4 : place * 8, halves ? half + place * 4 : place * 8 + 4}, angle = place * 4;
  auto kind_of = [&](int group) { return group < a.groups[0] ? 0 : group < a.groups[1] ? 1 : 2; };
  auto head_of = [&](int group, int kind) { return (group - (kind ? a.groups[kind - 1] : 0)) * kGroup + mine; };
  auto fetch = [&](int group, uint4* raw) {
    const int kind = kind_of(group), h = head_of(group, kind), heads = kind ? a.Hk : a.H;
    const T* p = (const T*)a.src[kind] + i * a.ss[kind][0] + h * a.ss[kind][1];
    const long long step = kHeads * a.ss[kind][1];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (h + u * kHeads < heads) {
        const uint2 x = __ldcs(reinterpret_cast<const uint2*>(p + u * step + at[0]));
        const uint2 y = __ldcs(reinterpret_cast<const uint2*>(p + u * step + at[1]));
        raw[u] = make_uint4(x.x, x.y, y.x, y.y);
      }
  };
  uint4 ahead[kUnroll] = {};
  fetch(split, ahead);
  const int deep = a.depth ? a.depth[i] : 0;
  const int b = row_of(c, i, lane);
  if (b < 0) return;
  int s, n, len;
  if (!row_span(c, b, s, n, len)) return;
  const int pos = len + i - s;
  if (a.cos && (a.depth ? deep < 0 || deep >= a.n_pos - len : pos >= a.n_pos)) return;
  const int turn = a.depth && a.cos ? len + deep : pos;  // whose angles
  const int page = page_of(c, b, pos);
  if (page < 0) return;
  const int off = pos & ((1 << c.log_page) - 1);
  Two wc[4], ws[4];  // w_i c and w_j s, s with the sign that it has for this value
  int kind = -1;
#pragma unroll 1
  for (int group = split; group < a.groups[2]; group += a.splits) {
    uint4 raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) raw[u] = ahead[u];
    if (group + a.splits < a.groups[2]) fetch(group + a.splits, ahead);
    const bool changed = kind != kind_of(group);
    kind = kind_of(group);
    const int h = head_of(group, kind), heads = kind ? a.Hk : a.H;
    T* dst = (T*)a.dst[kind];
    dst += kind ? page * a.ps[kind - 1][0] + off * a.ps[kind - 1][1] + h * a.ps[kind - 1][2] : i * a.qos[0] + h * a.qos[1];
    const long long step = kHeads * (kind ? a.ps[kind - 1][2] : a.qos[1]);
    auto store = [&](int u, const uint4& x) {
      if (h + u * kHeads >= heads) return;
      *reinterpret_cast<uint2*>(dst + u * step + at[0]) = make_uint2(x.x, x.y);
      *reinterpret_cast<uint2*>(dst + u * step + at[1]) = make_uint2(x.z, x.w);
    };
    if (kind == 2) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) store(u, raw[u]);
      continue;
    }
    const T* w = (const T*)a.w[kind];
    if (changed) {
      float wt[8], c4[4] = {1.f, 1.f, 1.f, 1.f}, s4[4] = {};
#pragma unroll
      for (int j = 0; j < 8; ++j) wt[j] = 1.f;
      if (w) {
        const uint2 x = *reinterpret_cast<const uint2*>(w + at[0]), y = *reinterpret_cast<const uint2*>(w + at[1]);
        unpack8<T>(make_uint4(x.x, x.y, y.x, y.y), wt);
      }
      if (turned) {
        const float4 x = *reinterpret_cast<const float4*>(a.cos + (long long)turn * half + angle);
        const float4 y = *reinterpret_cast<const float4*>(a.sin + (long long)turn * half + angle);
        c4[0] = x.x, c4[1] = x.y, c4[2] = x.z, c4[3] = x.w;
        s4[0] = y.x, s4[1] = y.y, s4[2] = y.z, s4[3] = y.w;
      }
#pragma unroll
      for (int j = 0; j < 8; j += 2) {  // (values j and j + 1)
        if (a.pairs) {
          wc[j / 2] = Two{wt[j] * c4[j / 2], wt[j + 1] * c4[j / 2]};
          ws[j / 2] = Two{-wt[j + 1] * s4[j / 2], wt[j] * s4[j / 2]};
        } else {
          const int m = j & 3;
          const float sign = j < 4 ? -1.f : 1.f;
          wc[j / 2] = Two{wt[j] * c4[m], wt[j + 1] * c4[m + 1]};
          ws[j / 2] = Two{sign * wt[j ^ 4] * s4[m], sign * wt[(j ^ 4) + 1] * s4[m + 1]};
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float v[8];
      unpack8<T>(raw[u], v);
      Two x[4], z[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = Two{v[2 * j], v[2 * j + 1]}, z[j] = mul2(x[j], wc[j]);
      if (turned) {  // (a value that is not turned has no partner to get an infinity from)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = fma2(a.pairs ? Two{x[j].y, x[j].x} : x[j ^ 2], ws[j], z[j]);
      }
      if (w) {
        Two s2 = mul2(x[0], x[0]);
#pragma unroll
        for (int j = 1; j < 4; ++j) s2 = fma2(x[j], x[j], s2);
        float sum = s2.x + s2.y;
#pragma unroll
        for (int o = kLanes / 2; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        const float r = rsqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = mul2(z[j], Two{r, r});
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) v[2 * j] = z[j].x, v[2 * j + 1] = z[j].y;
      store(u, pack8<T>(v));
    }
  }
}

}  // namespace
}  // namespace grid

using namespace grid;

static int append(const char* name, const grid_kv* kv, const grid_kv_chunk* chunk, const grid_heads* k, const grid_heads* v,
                  const grid_heads* q, const grid_heads* q_out, const grid_rotation* rot, const grid_head_norm* norm,
                  const int32_t* d_depth, int32_t* d_status, void* stream) {
  auto refuse = [&](int code, const char* why) { return set_error(code, std::string(name) + ": " + why); };
  AppendArgs a = {};
  if (!kv || !d_status || !make_chunk(kv, chunk, a.c) || (chunk->n_tokens && (!heads_ok(k) || !heads_ok(v))) ||
      (q != nullptr) != (q_out != nullptr) || (q && chunk->n_tokens && (!heads_ok(q) || !heads_ok(q_out))))
    return refuse(GRID_E_INVALID_ARG, "bad arguments");
  if (rot && (!rot->d_cos || !rot->d_sin || (uintptr_t)rot->d_cos % 16 || (uintptr_t)rot->d_sin % 16 ||
              rot->n_pos <= 0 || rot->rot <= 0 || rot->rot % 16 || rot->rot > kv->p.head_dim))
    return refuse(GRID_E_INVALID_ARG, "bad rotation (rot is a multiple of 16 up to head_dim)");
  if (norm && ((uintptr_t)norm->d_q % 16 || (uintptr_t)norm->d_k % 16 || !(norm->eps >= 0.f)))
    return refuse(GRID_E_INVALID_ARG, "bad norm");
  if (chunk->B > 65535) return refuse(GRID_E_TOO_LARGE, "more than 65535 rows");
  const grid_kv_pages& p = kv->p;
  auto heads = [&](int kind, const grid_heads* h, int count) {
    if (chunk->n_tokens && h) a.src[kind] = h->d, a.ss[kind][0] = h->token_stride, a.ss[kind][1] = h->head_stride;
    a.groups[kind] = (kind ? a.groups[kind - 1] : 0) + (h ? (count + kGroup - 1) / kGroup : 0);
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
  a.status = d_status, a.depth = d_depth;
  // (whole tokens where their warps fill the SMs anyway: as many as the registers let an SM hold.  32 trees of up to 64 tokens
  // in 128-wide heads 5.9 us, 7.1 with 32 warps for an SM)
  a.splits = std::max(1, std::min(a.groups[2], (p.head_dim == 128 ? 24 : 32) * kv->sms / std::max(1, chunk->n_tokens)));
  const long long blocks = ((long long)chunk->n_tokens * a.splits + kAppendWarps - 1) / kAppendWarps;
  const int rows = (chunk->B + kAppendWarps - 1) / kAppendWarps;
  if (blocks + rows > INT32_MAX) return refuse(GRID_E_TOO_LARGE, "too many head vectors in one call");
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

extern "C" int grid_kv_append(const grid_kv* kv, const grid_kv_chunk* chunk, const grid_heads* k, const grid_heads* v,
                              const grid_heads* q, const grid_heads* q_out, const grid_rotation* rot,
                              const grid_head_norm* norm, int32_t* d_status, void* stream) {
  return append("grid_kv_append", kv, chunk, k, v, q, q_out, rot, norm, nullptr, d_status, stream);
}

extern "C" int grid_kv_append_tree(const grid_kv* kv, const grid_kv_chunk* chunk, const grid_heads* k, const grid_heads* v,
                                   const grid_heads* q, const grid_heads* q_out, const grid_rotation* rot,
                                   const grid_head_norm* norm, const int32_t* d_depth, int32_t* d_status, void* stream) {
  return append("grid_kv_append_tree", kv, chunk, k, v, q, q_out, rot, norm, d_depth, d_status, stream);
}
