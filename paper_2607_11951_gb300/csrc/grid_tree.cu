// A row's chunk as a tree of drafted tokens: depths and visibility from the
// parents (grid_tree_plan), and the path that the sampled tokens take
// (grid_tree_accept).
#include "grid_model.cuh"

namespace grid {
namespace {

constexpr int kMaxWords = 32;  // 1,024 tokens of a row
constexpr int kPlanThreads = 128, kAcceptWarps = 4;

// Row b's tokens [a, a + n); false where they are not in order.
__device__ __forceinline__ bool tree_span(const grid_tree& t, int b, int& a, int& n) {
  a = t.d_start ? t.d_start[b] : b * (t.n_tokens / t.B);
  const int z = t.d_start ? t.d_start[b + 1] : a + t.n_tokens / t.B;
  n = z - a;
  return a >= 0 && z >= a && z <= t.n_tokens;
}

// A block per row.  A thread makes one word of one token's visibility by going up
// the tree in shared memory; the words of a token repeat the walk, so that none
// waits for another, and stop where the ancestors (in falling order) are below
// their bits.  Time is the chain of loads: the row's span, its parents, the walk
// (32 trees of up to 64 tokens: 1.7 us; one of eight 1.3).  The walks of deep trees
// are long, and there is one for each word of each token: a chain of 64 tokens
// takes 3.2 us, of 128 10.5, of 256 62, of 512 446, of 1,024 3,446 (random trees of
// these sizes 1.6, 2.8, 8.6, 26 and 98).
__global__ void __launch_bounds__(kPlanThreads) k_plan(const grid_tree tree, int32_t* __restrict__ depth,
                                                       uint32_t* __restrict__ sees, int words, int32_t* __restrict__ status) {
  __shared__ int16_t up[kMaxWords * 32];
  const int b = blockIdx.x, tid = threadIdx.x;
  pdl_wait();
  pdl_next();
  int a, n;
  const bool fits = tree_span(tree, b, a, n) && n <= 32 * words;
  if (!fits) {
    if (tid == 0) status[b] = GRID_ST_TREE;
    return;
  }
  bool ok = true;
  for (int i = tid; i < n; i += kPlanThreads) {
    const int p = tree.d_parent[a + i];
    ok = ok && p >= -1 && p < i;
    up[i] = (int16_t)p;
  }
  ok = __syncthreads_and(ok);
  if (tid == 0) status[b] = ok ? GRID_ST_OK : GRID_ST_TREE;
  for (int x = tid; x < n * words; x += kPlanThreads) {
    const int i = x / words, w = x - i * words;
    uint32_t bits = 0;
    int d = -1;
    for (int j = i; j >= (w ? 32 * w : 0); j = ok ? up[j] : -1) {  // (word 0 goes up to the root: it counts)
      if (j >> 5 == w) bits |= 1u << (j & 31);
      ++d;
    }
    sees[(long long)(a + i) * words + w] = bits;
    if (w == 0) depth[a + i] = d;
  }
}

// A warp per row.  The first kHeld * 32 tokens of the row (all of them, as a rule) are
// in registers, with what was sampled at them, so that a step down the tree is a
// compare, a ballot and a few shuffles; later ones are loaded in every step (256 trees
// of up to 64 tokens, paths of up to nine: 2.7 us; one 1.4).
constexpr int kHeld = 4;
__global__ void __launch_bounds__(kAcceptWarps * 32) k_accept(const grid_tree tree, const int32_t* __restrict__ tokens,
                                                              const int32_t* __restrict__ sampled, int eos, int most,
                                                              int32_t* __restrict__ path, int32_t* __restrict__ count,
                                                              int32_t* __restrict__ out, int32_t* __restrict__ status) {
  const int lane = threadIdx.x & 31, b = blockIdx.x * kAcceptWarps + (threadIdx.x >> 5);
  if (b >= tree.B) return;
  pdl_wait();
  pdl_next();
  int a, n;
  const bool fits = tree_span(tree, b, a, n);
  int parent[kHeld], token[kHeld], drawn[kHeld];
#pragma unroll
  for (int x = 0; x < kHeld; ++x) {
    const int j = 32 * x + lane;
    const bool in = fits && j < n;
    parent[x] = in ? tree.d_parent[a + j] : -2;
    token[x] = in ? tokens[a + j] : 0;
    drawn[x] = in ? sampled[a + j] : -1;
  }
  path += (long long)b * most;
  out += (long long)b * most;
  int node = fits && n > 0 ? 0 : -1, d = 0;
  bool ended = false;
  while (node >= 0 && d < most) {
    int t = -1;
#pragma unroll
    for (int x = 0; x < kHeld; ++x) {
      const int y = __shfl_sync(~0u, drawn[x], node & 31);
      if (node >> 5 == x) t = y;
    }
    if (node >= 32 * kHeld) t = sampled[a + node];
    if (lane == 0) {
      path[d] = node;
      out[d] = t;
    }
    ++d;
    ended = eos >= 0 && t == eos;
    if (ended || t < 0) break;
    int child = -1;
#pragma unroll
    for (int x = 0; x < kHeld; ++x) {  // (children come after their parent)
      const unsigned hit = __ballot_sync(~0u, parent[x] == node && token[x] == t && 32 * x + lane > node);
      if (child < 0 && hit) child = 32 * x + __ffs(hit) - 1;
    }
    for (int j = 32 * kHeld; child < 0 && j < n; j += 32) {
      const bool in = j + lane < n && j + lane > node;
      const unsigned hit = __ballot_sync(~0u, in && tree.d_parent[a + j + lane] == node && tokens[a + j + lane] == t);
      if (hit) child = j + __ffs(hit) - 1;
    }
    node = child;
  }
  for (int x = d + lane; x < most; x += 32) path[x] = out[x] = -1;
  if (lane == 0) {
    count[b] = d;
    status[b] = !fits ? GRID_ST_TREE : ended ? GRID_ST_COMPLETE : GRID_ST_OK;
  }
}

bool tree_ok(const grid_tree* t) {
  return t && t->B > 0 && t->n_tokens >= 0 && (t->d_parent || !t->n_tokens) && (t->d_start || t->n_tokens % t->B == 0);
}

}  // namespace
}  // namespace grid

using namespace grid;

extern "C" int grid_tree_plan(const grid_tree* tree, int32_t* d_depth, uint32_t* d_sees, int32_t n_words, int32_t* d_status,
                              void* stream) {
  if (!tree_ok(tree) || !d_status || n_words <= 0 || (tree->n_tokens && (!d_depth || !d_sees)))
    return set_error(GRID_E_INVALID_ARG, "grid_tree_plan: bad arguments");
  if (tree->B > 65535 || n_words > kMaxWords)
    return set_error(GRID_E_TOO_LARGE, "grid_tree_plan: more than 65535 rows or 32 words");
  GRID_CUDA(launch_pdl(k_plan, dim3((unsigned)tree->B), dim3(kPlanThreads), 0, (cudaStream_t)stream, *tree, d_depth, d_sees, n_words, d_status));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}

extern "C" int grid_tree_accept(const grid_tree* tree, const int32_t* d_tokens, const int32_t* d_sampled, int32_t eos,
                                int32_t max_path, int32_t* d_path, int32_t* d_count, int32_t* d_out, int32_t* d_status,
                                void* stream) {
  if (!tree_ok(tree) || (tree->n_tokens && (!d_tokens || !d_sampled)) || max_path <= 0 || !d_path || !d_count || !d_out ||
      !d_status)
    return set_error(GRID_E_INVALID_ARG, "grid_tree_accept: bad arguments");
  if (tree->B > 65535) return set_error(GRID_E_TOO_LARGE, "grid_tree_accept: more than 65535 rows");
  GRID_CUDA(launch_pdl(k_accept, dim3((unsigned)((tree->B + kAcceptWarps - 1) / kAcceptWarps)), dim3(kAcceptWarps * 32), 0,
                       (cudaStream_t)stream, *tree, d_tokens, d_sampled, eos, max_path, d_path, d_count, d_out, d_status));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}
