// Shared by the paged cache's append and attention: the chunk as the kernels
// take it, the checks of a row, head vectors in 16-byte pieces, and the object
// behind the handle.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "grid_model.cuh"

namespace grid {

struct Chunk {  // grid_kv_chunk with the cache's geometry
  const int32_t* table;
  const int32_t* len;
  const int32_t* start;
  long long table_stride;
  int max_pages, B, N, n_pages, log_page, T;  // T: tokens of every row where start is NULL
  int max_n;  // the most tokens of a row
};

// Row b's tokens [a, a + n) and its first position; false where they are not in order.
__device__ __forceinline__ bool row_span(const Chunk& c, int b, int& a, int& n, int& len) {
  a = c.start ? c.start[b] : b * c.T;
  const int z = c.start ? c.start[b + 1] : a + c.T;
  len = c.len[b];
  n = z - a;
  return a >= 0 && z >= a && z <= c.N && n <= c.max_n && len >= 0 && (long long)len + n <= (long long)c.max_pages << c.log_page;
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

inline bool heads_ok(const grid_heads* h) {
  return h && h->d && (uintptr_t)h->d % 16 == 0 && h->token_stride >= 0 && h->head_stride >= 0 &&
         h->token_stride % 8 == 0 && h->head_stride % 8 == 0;
}

}  // namespace grid

struct grid_kv {
  grid_kv_pages p;
  int* gave_up = nullptr;    // one word on the device: a wait of an attend ran out (the first field after p: tests set it)
  int log_page = 0, sms = 152;
  CUtensorMap k_map, v_map;  // of the pools, for the attention's tiles
  float* parts = nullptr;    // partial results of the attention's split rows
  float2* part_ml = nullptr;
  int* joined = nullptr;
  grid::Arena mem;
};

// The chunk as the kernels take it; false where its arguments are bad.
inline bool make_chunk(const grid_kv* kv, const grid_kv_chunk* ch, grid::Chunk& c) {
  if (!ch || !ch->d_table || !ch->d_len || ch->B <= 0 || ch->n_tokens < 0 || ch->max_pages <= 0 ||
      ch->table_stride < ch->max_pages || ((int64_t)ch->max_pages << kv->log_page) > INT32_MAX ||
      (!ch->d_start && ch->n_tokens % ch->B))
    return false;
  c = grid::Chunk{ch->d_table, ch->d_len, ch->d_start, ch->table_stride, ch->max_pages, ch->B, ch->n_tokens,
            kv->p.n_pages, kv->log_page, ch->n_tokens / ch->B, INT32_MAX};
  return true;
}
