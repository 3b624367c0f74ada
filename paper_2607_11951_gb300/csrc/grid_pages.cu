// The pages of a paged cache: the next step's table from the present one
// (grid_pages_update), copies of pages that are held in part (grid_kv_copy), and
// an accepted path's keys and values moved next to what is cached
// (grid_kv_compact).
#include <climits>
#include <new>

#include "grid_kv.cuh"

namespace grid {
namespace {

// ---------------------------------------------------------------------------
// The update counts, for every page, the new rows that keep it whole, finds the
// row that a page in part stays with, ranks the free pages by prefix sums and
// deals them out: five steps, each of which needs all of the one before, and a
// launch costs more than a step.  Up to 1,024 rows and 16,384 pages are one
// block, a thread per row, the pages' counts in its shared memory; more are a
// cluster of eight blocks, whose barriers order what they wrote to memory.
// Counts are atomic additions and minima of integers: their order changes
// nothing.  Bound by the chains of loads, in one block by its instructions, and in
// the cluster by an atomic addition in L2 for each entry of the table, issued by
// eight SMs: four rows and 56 pages 3.9 us (as a cluster 9.1), 256 rows of up to 32
// of 3,148 pages 7.4 (10.9), 30 of up to 1,001 of 10,419 13.2 (20.7), 1,000 of up to
// 32 of 12,276 18.0 (20.0), 256 of up to 126 of 11,279 14.6 (13.2: the table's
// entries count as well, but the rule goes by what one block has room for); 256 of
// up to 1,001 of 87,348 (a cluster) take 34 to 48, by how the pages lie.
constexpr int kUpdateThreads = 1024, kUpdateBlocks = 8;
constexpr int kAlonePages = 16384;
constexpr int kMostPages = 1 << 30;  // (so that an index past the last page by a stride is still one)

struct UpdateArgs {
  grid_pages_step s;
  int n_pages, log_page;
  int *owner, *fresh;  // [n_pages]: the lowest row that keeps the page in part; the free pages in their order
};

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_rank() {
  int r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// The int at x of block r's shared memory.
__device__ __forceinline__ int from_block(const int* x, int r) {
  uint32_t at;
  int v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(x)), "r"(r));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
// The sum over the block's threads before this one, and over all of them.
__device__ __forceinline__ int before(int x, int* sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int pre = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(~0u, pre, o);
    if (lane >= o) pre += y;
  }
  if (lane == 31) sums[warp] = pre;
  __syncthreads();
  if (warp == 0) {
    int y = lane < (int)blockDim.x / 32 ? sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int z = __shfl_up_sync(~0u, y, o);
      if (lane >= o) y += z;
    }
    sums[lane] = y;
  }
  __syncthreads();
  total = sums[31];
  pre += (warp ? sums[warp - 1] : 0) - x;
  __syncthreads();
  return pre;
}

__device__ __forceinline__ int pages_for(const UpdateArgs& u, int tokens) {
  return (int)(((long long)tokens + (1 << u.log_page) - 1) >> u.log_page);
}

__global__ void __launch_bounds__(kUpdateThreads) k_update(const UpdateArgs u) {
  constexpr int blocks = kUpdateBlocks;
  const grid_pages_step& s = u.s;
  __shared__ int sums[32], free_here;
  const int tid = threadIdx.x, lane = tid & 31, rank = cluster_rank();
  const int threads = blocks * kUpdateThreads, at = rank * kUpdateThreads + tid;
  const int warps = threads / 32, warp = at / 32;
  // (between the steps: the page in part that has to be copied, the fresh pages before the row's; d_status is what the row keeps,
  // or ~ that where it is not valid or its row of the new table too short; d_held_out may be d_want and is written last)
  int32_t *from = s.d_copies, *to = from + s.B, *tokens = to + s.B;
  auto sync = [&]() {
    __syncwarp();
    cluster_sync();
  };
  pdl_wait();
  pdl_next();
#pragma unroll 4
  for (int p = at; p < u.n_pages; p += threads) {
    s.d_refs[p] = 0;
    u.owner[p] = INT_MAX;
  }
  sync();
  // ---- a warp per row: whole pages are counted, pages in part look for their row
  for (int b = warp; b < s.B; b += warps) {
    const int parent = s.d_parent ? s.d_parent[b] : b, want = s.d_want[b];
    bool ok = parent >= -1 && parent < s.A;
    const int held = ok && parent >= 0 ? s.d_held[parent] : 0;
    int keep = ok && parent >= 0 ? (s.d_keep ? s.d_keep[b] : held) : 0;
    const int32_t* old = s.d_table + (ok && parent >= 0 ? parent * s.table_stride : 0);
    int32_t* out = s.d_table_out + b * s.table_out_stride;
    ok = ok && keep >= 0 && keep <= held && want >= keep && pages_for(u, keep) <= min(s.width, s.width_out);
    const int all = ok ? pages_for(u, keep) : 0;
#pragma unroll 8
    for (int j = lane; j < all; j += 32) {
      const int p = old[j];
      ok = ok && p >= 0 && p < u.n_pages;
    }
    ok = __all_sync(~0u, ok);
    if (!ok) keep = 0;
    const int full = keep >> u.log_page, kept = pages_for(u, keep);
    int last = -1;
#pragma unroll 8
    for (int j = lane; j < s.width_out; j += 32) {
      const int p = j < kept ? old[j] : -1;
      out[j] = p;
      if (j < full)
        atomicAdd(&s.d_refs[p], 1);
      else if (j < kept)
        atomicMin(&u.owner[p], b), last = p;
    }
    last = __reduce_max_sync(~0u, last);
    if (lane == 0) {
      const bool room = pages_for(u, want) <= s.width_out;
      from[b] = last;
      to[b] = ok && room ? pages_for(u, want) - full : 0;
      s.d_status[b] = ok && room ? keep : ~keep;
    }
  }
  sync();
  // ---- a thread per row, of one block: who keeps a page in part, and how many fresh pages the rows before take
  if (rank == 0) {
    const int per = (s.B + kUpdateThreads - 1) / kUpdateThreads, b0 = tid * per, b1 = min(s.B, b0 + per);
    int sum = 0;
    for (int b = b0; b < b1; ++b) {
      const int last = __ldcg(from + b);
      const bool stays = last >= 0 && __ldcg(u.owner + last) == b && __ldcg(s.d_refs + last) == 0 && !(s.d_pinned && s.d_pinned[last]);
      if (stays) {  // (no other row with this page in part may, whatever it reads here)
        s.d_refs[last] = 1;
        from[b] = -1;
      }
      const int need = max(0, __ldcg(to + b) - stays);
      tokens[b] = need;
      sum += need;
    }
    int all;
    int pre = before(sum, sums, all);
    for (int b = b0; b < b1; ++b) {
      to[b] = pre;
      pre += tokens[b];
    }
  }
  sync();
  // ---- the free pages in their order: 32 at a time, a run of them to a warp
  const int run = ((u.n_pages + warps - 1) / warps + 31) & ~31;
  const int p0 = min((long long)u.n_pages, (long long)warp * run), p1 = min((long long)u.n_pages, (long long)p0 + run);
  auto free_of = [&](int p) {
    return __ballot_sync(~0u, p + lane < p1 && __ldcg(s.d_refs + p + lane) == 0 && !(s.d_pinned && s.d_pinned[p + lane]));
  };
  int n = 0;
#pragma unroll 4
  for (int p = p0; p < p1; p += 32) n += __popc(free_of(p));
  int here;
  int pre = before(lane == 0 ? n : 0, sums, here);
  pre = __shfl_sync(~0u, pre, 0);
  if (tid == 0) free_here = here;
  sync();
  int all = 0;
  for (int r = 0; r < blocks; ++r) {
    const int x = from_block(&free_here, r);
    if (r < rank) pre += x;
    all += x;
  }
#pragma unroll 4
  for (int p = p0; p < p1; p += 32) {
    const unsigned bits = free_of(p);
    if (bits >> lane & 1) u.fresh[pre + __popc(bits & ((1u << lane) - 1))] = p + lane;
    pre += __popc(bits);
  }
  sync();
  // ---- a warp per row: its fresh pages
  for (int b = warp; b < s.B; b += warps) {
    const int state = s.d_status[b], keep = state >= 0 ? state : ~state, want = s.d_want[b];
    const int copied = __ldcg(from + b), first = __ldcg(to + b), need = __ldcg(tokens + b);
    const int full = keep >> u.log_page, part = keep & ((1 << u.log_page) - 1);
    const bool fits = state >= 0 && (need == 0 || first + need <= all);
    int32_t* out = s.d_table_out + b * s.table_out_stride;
    const int begin = full + (part && copied < 0);
    __syncwarp();
    if (fits) {
      for (int j = lane; j < need; j += 32) {
        const int p = __ldcg(u.fresh + first + j);
        out[begin + j] = p;
        s.d_refs[p] = 1;
        if (j == 0) to[b] = copied >= 0 ? p : -1;
      }
    } else if (lane == 0 && copied >= 0) {
      out[full] = -1;
    }
    if (lane == 0) {
      const bool copies = fits && copied >= 0;
      if (!copies) from[b] = to[b] = -1;
      tokens[b] = copies ? part : 0;
      s.d_held_out[b] = fits ? want : copied >= 0 ? full << u.log_page : keep;
      s.d_status[b] = fits ? GRID_ST_OK : GRID_ST_PAGES;
    }
  }
}

// One block: a thread per row, then a thread per entry of the table (a warp per row would be five times the instructions, for
// rows of a dozen pages); counts in shared memory.
struct UpdateRow {
  int parent, keep, want, kept;  // kept: pages, that in part too; -1: not valid
  int last, first;               // its page in part (that has to be copied, later on), the fresh pages of the rows before it
};
constexpr unsigned kPinned = 1u << 31;  // (in a page's count)
__global__ void __launch_bounds__(kUpdateThreads) k_update_alone(const UpdateArgs u) {
  const grid_pages_step& s = u.s;
  extern __shared__ __align__(16) uint8_t raw[];
  UpdateRow* const rows = reinterpret_cast<UpdateRow*>(raw);
  unsigned* const refs = reinterpret_cast<unsigned*>(rows + s.B);
  int* const owner = reinterpret_cast<int*>(refs + u.n_pages);  // then the free pages in their order
  __shared__ int sums[32], bad;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = tid;
  pdl_wait();
  pdl_next();
  UpdateRow r = {};
  if (b < s.B) {
    r.parent = s.d_parent ? s.d_parent[b] : b, r.want = s.d_want[b];
    r.keep = s.d_keep ? s.d_keep[b] : INT_MAX;
  }
#pragma unroll 4
  for (int p = tid; p < u.n_pages; p += kUpdateThreads) {
    refs[p] = s.d_pinned && s.d_pinned[p] ? kPinned : 0u;
    owner[p] = INT_MAX;
  }
  if (tid == 0) bad = 0;
  if (b < s.B) {
    const bool some = r.parent >= 0 && r.parent < s.A;
    const int held = some ? s.d_held[r.parent] : 0;
    if (!some) r.keep = 0;
    if (some && !s.d_keep) r.keep = held;
    const bool ok = (some || r.parent == -1) && r.keep >= 0 && r.keep <= held && r.want >= r.keep &&
                    pages_for(u, r.keep) <= min(s.width, s.width_out);
    if (!ok) r.keep = 0;
    r.kept = ok ? pages_for(u, r.keep) : -1;
    r.last = -1;
    rows[b] = r;
  }
  __syncthreads();
  // ---- whole pages are counted, pages in part noted
  {
    // (a thread's entries are kUpdateThreads apart: rows and columns by addition, four loads at once)
    const int w = s.width_out, rows_on = kUpdateThreads / w, on = kUpdateThreads - rows_on * w;
    int i = tid / w, j = tid - i * w;
    constexpr int kAtOnce = 4;
    while (i < s.B) {
      int at_i[kAtOnce], at_j[kAtOnce], p[kAtOnce];
#pragma unroll
      for (int y = 0; y < kAtOnce; ++y) {
        at_i[y] = i, at_j[y] = j;
        p[y] = -1;
        if (i < s.B && j < rows[i].kept) p[y] = s.d_table[rows[i].parent * s.table_stride + j];
        i += rows_on, j += on;
        if (j >= w) j -= w, ++i;
      }
#pragma unroll
      for (int y = 0; y < kAtOnce; ++y) {
        if (at_i[y] >= s.B) break;
        s.d_table_out[at_i[y] * s.table_out_stride + at_j[y]] = p[y];
        UpdateRow& row = rows[at_i[y]];
        if (at_j[y] >= row.kept) continue;
        if (p[y] < 0 || p[y] >= u.n_pages)
          bad = 1;
        else if (at_j[y] < row.keep >> u.log_page)
          atomicAdd(&refs[p[y]], 1u);
        else
          row.last = p[y];
      }
    }
  }
  __syncthreads();
  if (bad)  // (rows with a page outside the pool take back what they counted)
    for (int i = warp; i < s.B; i += kUpdateThreads / 32) {
      const int kept = rows[i].kept;
      const int32_t* old = s.d_table + (kept > 0 ? rows[i].parent * s.table_stride : 0);
      bool ok = true;
      for (int j = lane; j < kept; j += 32) ok = ok && old[j] >= 0 && old[j] < u.n_pages;
      if (__all_sync(~0u, ok)) continue;
      for (int j = lane; j < kept; j += 32) {
        const int p = old[j];
        s.d_table_out[i * s.table_out_stride + j] = -1;
        if (p >= 0 && p < u.n_pages && j < rows[i].keep >> u.log_page) atomicSub(&refs[p], 1u);
      }
      __syncwarp();
      if (lane == 0) rows[i].kept = -1, rows[i].keep = 0, rows[i].last = -1;
    }
  if (bad) __syncthreads();
  if (b < s.B) r = rows[b];
  if (b < s.B && r.last >= 0) atomicMin(&owner[r.last], b);
  __syncthreads();
  // ---- who keeps a page in part, and how many fresh pages the rows before take
  bool room = false;
  int need = 0, full = 0;
  if (b < s.B) {
    full = r.keep >> u.log_page;
    const bool stays = r.last >= 0 && owner[r.last] == b && refs[r.last] == 0;
    // (its own thread alone writes this count; another row that has the page in part is not its owner, whatever it reads)
    if (stays) refs[r.last] = 1, r.last = -1;
    room = r.kept >= 0 && pages_for(u, r.want) <= s.width_out;
    need = room ? pages_for(u, r.want) - full - stays : 0;
  }
  int wanted, all;
  const int first = before(need, sums, wanted);
  if (b < s.B) rows[b].first = first, rows[b].last = r.last;
  // ---- the free pages in their order: 32 at a time, a run of them to a warp
  const int run = ((u.n_pages + kUpdateThreads - 1) / kUpdateThreads) * 32;
  const int p0 = min(u.n_pages, warp * run), p1 = min(u.n_pages, p0 + run);
  int n = 0;
  for (int p = p0; p < p1; p += 32) n += __popc(__ballot_sync(~0u, p + lane < p1 && refs[p + lane] == 0));
  int pre = before(lane == 0 ? n : 0, sums, all);
  pre = __shfl_sync(~0u, pre, 0);
  for (int p = p0; p < p1; p += 32) {  // (nobody looks for an owner any more)
    const unsigned bits = __ballot_sync(~0u, p + lane < p1 && refs[p + lane] == 0);
    if (bits >> lane & 1) owner[pre + __popc(bits & ((1u << lane) - 1))] = p + lane;
    pre += __popc(bits);
  }
  __syncthreads();
  // ---- a thread per fresh page: its row is the last one that begins at or before it
  for (int x = tid; x < min(wanted, all); x += kUpdateThreads) {
    int i = 0;
    for (int step = kUpdateThreads / 2; step; step /= 2)
      if (i + step < s.B && rows[i + step].first <= x) i += step;
    const int end = i + 1 < s.B ? rows[i + 1].first : wanted;
    if (end > all) continue;  // (not all of the row's are there)
    const int whole = rows[i].keep >> u.log_page, stays = (rows[i].keep & ((1 << u.log_page) - 1)) && rows[i].last < 0;
    const int p = owner[x];
    s.d_table_out[i * s.table_out_stride + whole + stays + x - rows[i].first] = p;
    refs[p] = 1;
  }
  if (b < s.B) {
    const bool fits = room && (need == 0 || first + need <= all), copies = fits && r.last >= 0;
    if (!fits && r.last >= 0) s.d_table_out[b * s.table_out_stride + full] = -1;
    s.d_copies[b] = copies ? r.last : -1;
    s.d_copies[s.B + b] = copies ? owner[first] : -1;
    s.d_copies[2 * s.B + b] = copies ? r.keep & ((1 << u.log_page) - 1) : 0;
    s.d_held_out[b] = fits ? r.want : r.last >= 0 ? full << u.log_page : r.keep;
    s.d_status[b] = fits ? GRID_ST_OK : GRID_ST_PAGES;
  }
  __syncthreads();
  for (int p = tid; p < u.n_pages; p += kUpdateThreads) s.d_refs[p] = refs[p] & ~kPinned;
}

// ---------------------------------------------------------------------------
// A copy's tokens, in pieces of 16 bytes.  What lies side by side (all of them, or a
// head's) is cut into chunks of kAhead pieces a thread, which are loaded at once;
// the chunks of a copy and pool go to `splits` blocks in turn.  128 copies of some
// 32 tokens (8 heads of 128, 29 MB moved) take 6.5 us, 4.5 TB/s (256 threads 7.2;
// two or eight pieces a thread 6.6 to 7.2); three of a few tokens 1.5.  Pieces
// are counted in 32 bits, up to kMostPieces (16 GB) of a page.
constexpr int kCopyThreads = 128, kAhead = 4, kChunk = kCopyThreads * kAhead;
constexpr int64_t kMostPieces = 1 << 30;

struct CopyArgs {
  uint4* pool[2];
  long long page[2], token[2], head[2];  // strides in pieces
  const int32_t* copies;
  int32_t* status;
  int n, n_pages, page_size, Hk, log_parts, splits;
};

__global__ void __launch_bounds__(kCopyThreads) k_copy(const CopyArgs c) {
  const int i = blockIdx.x / (2 * c.splits), rest = blockIdx.x - i * 2 * c.splits, kv = rest & 1, split = rest >> 1;
  pdl_wait();
  pdl_next();
  const int src = c.copies[i], dst = c.copies[c.n + i], tokens = c.copies[2 * c.n + i];
  const bool none = src < 0, ok = none || (src < c.n_pages && dst >= 0 && dst < c.n_pages && tokens >= 0 && tokens <= c.page_size);
  if (rest == 0 && threadIdx.x == 0) c.status[i] = ok ? GRID_ST_OK : GRID_ST_PAGES;
  if (none || !ok || src == dst) return;
  const long long page = kv ? c.page[1] : c.page[0], token = kv ? c.token[1] : c.token[0], head = kv ? c.head[1] : c.head[0];
  const int parts = 1 << c.log_parts;
  const bool whole = head == parts && token == (long long)c.Hk << c.log_parts;  // tokens side by side, their heads too
  const int run = (whole ? tokens * c.Hk : tokens) << c.log_parts, runs = whole ? 1 : c.Hk;
  const int per = (run + kChunk - 1) / kChunk;
  uint4* pool = kv ? c.pool[1] : c.pool[0];
  const uint4* from = pool + src * page;
  uint4* to = pool + dst * page;
  for (int k = split; k < runs * per; k += c.splits) {
    const int r = k / per, z0 = (k - r * per) * kChunk + threadIdx.x;
    auto place = [&](int z) { return whole ? (long long)z : r * head + (z >> c.log_parts) * token + (z & (parts - 1)); };
    uint4 v[kAhead];
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
      if (z0 + y * kCopyThreads < run) v[y] = from[place(z0 + y * kCopyThreads)];
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
      if (z0 + y * kCopyThreads < run) to[place(z0 + y * kCopyThreads)] = v[y];
  }
}

// ---------------------------------------------------------------------------
// A thread owns one 16-byte piece of a token's keys or values and takes it down
// the row's path: token j comes from path[j] >= j, so that what it writes has
// been read before, kSteps tokens at a time.  No other thread touches the piece.
// Time is the chain of loads: the row, its path, the pages, the pieces (256 paths
// of up to nine tokens, 8 heads of 128: 3.1 us; one path 1.7).
constexpr int kCompactThreads = 128, kSteps = 8;

struct CompactArgs {
  Chunk c;
  uint4* pool[2];
  long long page[2], token[2], head[2];
  const int32_t *path, *count;
  int32_t* status;
  int most, Hk, log_parts, blocks;  // blocks per row
};

__global__ void __launch_bounds__(kCompactThreads) k_compact(const CompactArgs a) {
  const int b = blockIdx.x / a.blocks, block = blockIdx.x - b * a.blocks, lane = threadIdx.x & 31;
  const Chunk& c = a.c;
  pdl_wait();
  pdl_next();
  const int32_t* path = a.path + (long long)b * a.most;
  const int count = a.count[b];
  int first, n, len;
  const bool row = row_span(c, b, first, n, len);
  // the lane's token of the path: checked by every warp for itself, 32 at a time
  bool tree = count >= 0 && count <= min(a.most, n), pages = row;
  if (row && tree)
    for (int j = lane; j < count; j += 32) {
      const int at = path[j], was = j ? path[j - 1] : -1;
      tree = tree && at > was && at >= 0 && at < n;
      if (tree) pages = pages && page_of(c, b, len + at) >= 0 && page_of(c, b, len + j) >= 0;
    }
  tree = __all_sync(~0u, tree), pages = __all_sync(~0u, pages);
  if (block == 0 && threadIdx.x == 0) a.status[b] = !row ? GRID_ST_PAGES : !tree ? GRID_ST_TREE : !pages ? GRID_ST_PAGES : GRID_ST_OK;
  if (!tree || !pages) return;
  const int piece = block * kCompactThreads + threadIdx.x, each = a.Hk << a.log_parts;  // pieces of a token's keys, or values
  const int kv = piece >= each, mine = piece - kv * each, mask = (1 << c.log_page) - 1;
  const bool in = piece < 2 * each;
  uint4* pool = a.pool[kv] + (mine >> a.log_parts) * a.head[kv] + (mine & ((1 << a.log_parts) - 1));
  for (int j0 = 0; j0 < count; j0 += 32) {
    const int j = j0 + lane, at = j < count ? path[j] : 0;
    const bool moved = j < count && at != j;
    const int p = moved ? page_of(c, b, len + at) : 0, q = moved ? page_of(c, b, len + j) : 0;
    unsigned left = __ballot_sync(~0u, moved);
    while (left) {
      uint4 v[kSteps];
      unsigned now = left;
#pragma unroll
      for (int y = 0; y < kSteps; ++y) {
        const int l = now ? __ffs(now) - 1 : 0;
        const int page = __shfl_sync(~0u, p, l), off = (len + __shfl_sync(~0u, at, l)) & mask;
        if (now && in) v[y] = pool[page * a.page[kv] + off * a.token[kv]];
        now &= now - 1;
      }
      now = left;
#pragma unroll
      for (int y = 0; y < kSteps; ++y) {
        const int l = now ? __ffs(now) - 1 : 0;
        const int page = __shfl_sync(~0u, q, l);
        if (now && in) pool[page * a.page[kv] + ((len + j0 + l) & mask) * a.token[kv]] = v[y];
        now &= now - 1;
      }
      left = now;
    }
  }
}

// The pools in pieces of 16 bytes.
template <typename Args>
void set_pools(const grid_kv* kv, Args& a) {
  const grid_kv_pages& p = kv->p;
  void* const d[2] = {p.d_k, p.d_v};
  const int64_t* const st[2] = {p.k_stride, p.v_stride};
  for (int i = 0; i < 2; ++i) {
    a.pool[i] = (uint4*)d[i];
    a.page[i] = st[i][0] / 8, a.token[i] = st[i][1] / 8, a.head[i] = st[i][2] / 8;
  }
  a.Hk = p.n_kv_heads;
  a.log_parts = p.head_dim == 64 ? 3 : 4;
}

}  // namespace
}  // namespace grid

using namespace grid;

struct grid_pages {
  int n_pages = 0, log_page = 0;
  int *owner = nullptr, *fresh = nullptr;
  Arena mem;
};

extern "C" int grid_pages_create(int32_t n_pages, int32_t page_size, grid_pages** out) {
  if (!out || n_pages <= 0 || page_size < 8 || page_size > 1024 || (page_size & (page_size - 1)))
    return set_error(GRID_E_INVALID_ARG, "grid_pages_create: n_pages is positive, page_size a power of two in 8 .. 1024");
  if (n_pages > kMostPages) return set_error(GRID_E_TOO_LARGE, "grid_pages_create: more than 2^30 pages");
  grid_pages* g = new (std::nothrow) grid_pages;
  if (!g) return set_error(GRID_E_TOO_LARGE, "grid_pages_create: out of host memory");
  g->n_pages = n_pages;
  while (1 << g->log_page < page_size) ++g->log_page;
  int rc = g->mem.alloc((size_t)n_pages * sizeof(int), (void**)&g->owner);
  if (!rc) rc = g->mem.alloc((size_t)n_pages * sizeof(int), (void**)&g->fresh);
  const cudaError_t e = rc ? cudaSuccess : cudaFuncSetAttribute(k_update_alone, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                               kUpdateThreads * sizeof(UpdateRow) + kAlonePages * 8);
  if (rc || e != cudaSuccess) {
    g->mem.release();
    delete g;
    return rc ? rc : set_error(GRID_E_CUDA, std::string("grid_pages_create: ") + cudaGetErrorString(e));
  }
  *out = g;
  return GRID_OK;
}

extern "C" void grid_pages_free(grid_pages* g) {
  if (!g) return;
  g->mem.release();
  delete g;
}

extern "C" int grid_pages_update(const grid_pages* g, const grid_pages_step* s, void* stream) {
  if (!g || !s || !s->d_table || !s->d_held || !s->d_want || !s->d_table_out || !s->d_held_out || !s->d_copies || !s->d_refs ||
      !s->d_status || s->A <= 0 || s->B <= 0 || s->width <= 0 || s->width_out <= 0 || s->table_stride < s->width ||
      s->table_out_stride < s->width_out || (!s->d_parent && s->B > s->A))
    return set_error(GRID_E_INVALID_ARG, "grid_pages_update: bad arguments");
  if (s->A > 65535 || s->B > 65535) return set_error(GRID_E_TOO_LARGE, "grid_pages_update: more than 65535 rows");
  if ((int64_t)s->B * s->width_out > INT32_MAX)
    return set_error(GRID_E_TOO_LARGE, "grid_pages_update: a table of more than 2^31 - 1 entries");
  UpdateArgs u = {*s, g->n_pages, g->log_page, g->owner, g->fresh};
  if (s->B <= kUpdateThreads && g->n_pages <= kAlonePages)
    GRID_CUDA(launch_pdl(k_update_alone, dim3(1), dim3(kUpdateThreads), s->B * sizeof(UpdateRow) + g->n_pages * 8, (cudaStream_t)stream, u));
  else
    GRID_CUDA(launch_cluster(k_update, dim3(kUpdateBlocks), dim3(kUpdateThreads), 0, kUpdateBlocks, (cudaStream_t)stream, u));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}

extern "C" int grid_kv_copy(const grid_kv* kv, const int32_t* d_copies, int32_t n, int32_t* d_status, void* stream) {
  if (!kv || !d_copies || !d_status || n <= 0) return set_error(GRID_E_INVALID_ARG, "grid_kv_copy: bad arguments");
  if (n > 65535) return set_error(GRID_E_TOO_LARGE, "grid_kv_copy: more than 65535 copies");
  if ((int64_t)kv->p.n_kv_heads * kv->p.page_size * kv->p.head_dim / 8 > kMostPieces)
    return set_error(GRID_E_TOO_LARGE, "grid_kv_copy: pages of more than 16 GB of keys");
  CopyArgs c = {};
  set_pools(kv, c);
  c.copies = d_copies, c.status = d_status, c.n = n;
  c.n_pages = kv->p.n_pages, c.page_size = kv->p.page_size;
  // (a block for each chunk of half a page, the usual copy; at most 64)
  const int half = (c.page_size / 2) << c.log_parts;
  const bool whole = c.head[0] == 1 << c.log_parts && c.token[0] == (long long)c.Hk << c.log_parts;
  c.splits = std::min<int64_t>(64, whole ? ((int64_t)half * c.Hk + kChunk - 1) / kChunk : (int64_t)c.Hk * ((half + kChunk - 1) / kChunk));
  GRID_CUDA(launch_pdl(k_copy, dim3((unsigned)(n * 2 * c.splits)), dim3(kCopyThreads), 0, (cudaStream_t)stream, c));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}

extern "C" int grid_kv_compact(const grid_kv* kv, const grid_kv_chunk* chunk, const int32_t* d_path, const int32_t* d_count,
                               int32_t max_path, int32_t* d_status, void* stream) {
  CompactArgs a = {};
  if (!kv || !d_path || !d_count || !d_status || max_path <= 0 || !make_chunk(kv, chunk, a.c))
    return set_error(GRID_E_INVALID_ARG, "grid_kv_compact: bad arguments");
  if (chunk->B > 65535) return set_error(GRID_E_TOO_LARGE, "grid_kv_compact: more than 65535 rows");
  if ((int64_t)2 * kv->p.n_kv_heads * kv->p.head_dim / 8 > kMostPieces)
    return set_error(GRID_E_TOO_LARGE, "grid_kv_compact: too many heads");
  set_pools(kv, a);
  a.path = d_path, a.count = d_count, a.status = d_status, a.most = max_path;
  a.blocks = ((2 * a.Hk << a.log_parts) + kCompactThreads - 1) / kCompactThreads;
  if ((int64_t)chunk->B * a.blocks > INT32_MAX) return set_error(GRID_E_TOO_LARGE, "grid_kv_compact: too many heads and rows");
  GRID_CUDA(launch_pdl(k_compact, dim3((unsigned)(chunk->B * a.blocks)), dim3(kCompactThreads), 0, (cudaStream_t)stream, a));
  GRID_CUDA(cudaGetLastError());
  return GRID_OK;
}
