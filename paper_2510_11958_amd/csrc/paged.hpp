// A paged key/value cache: requests keep their keys and values in pages of a shared pool, found through a block table per request.
// Here are the pages' bookkeeping (page_tables_kernel, page_rows_kernel), the append (paged_append_kernel) and what the attention kernels
// share; the attention itself is in attention_paged.hpp.
//
// Pool: K and V each [n_pages][n_kv_heads][page_size][head_dim], so that the keys of one head in one page are one contiguous run of
// page_size * head_dim elements (4 KiB at 16 keys of 128 bf16 values).  Page sizes are powers of two from 16 to 256: a group of 16 keys,
// which is what a wave of the attention kernels loads together, never leaves its page.
#pragma once
#include <limits.h>

#include "attention.hpp"
#include "gemv_mfma.hpp"

namespace dmtd {

constexpr int kPagedMaxRequests = 8192;      // requests of a call: their prefix sums lie in LDS

// What the append and the attention know of the cache
struct PagedView {
  void *k, *v;
  long page_stride;                 // elements from page to page
  const int* table;                 // [n_req][max_pages]
  int n_pages, page_shift, n_req, max_pages, nh, nkv, max_rows;
  int limit;                        // positions a request may have: the block table's, or the rotary table's where that is shorter
  int gq, gq_mul, rpb_few, rpb_tall;      // query heads per KV head, what a division by them is replaced by, rows of 16 and of 128 query vectors
  __device__ __forceinline__ int row_of(int v) const { return (v * gq_mul) >> 16; }      // v / gq for v < 128: gq_mul = 2^16 / gq + 1 is off by less than 1 / gq for those
};

// Sums over the lanes up to and with this one, without LDS: within rows of 16, then the rows' last values onto the rows behind them
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);      // row_shr:1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);      // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);      // row_bcast:31 into rows 2 and 3
  return v;
}

// Sum of v over the threads before this one, and over all of them, in a block of NT threads
template <int NT, typename T>
__device__ __forceinline__ T block_scan(T v, T* wave_sums /* LDS, NT / 64 */, T& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T incl = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T u = __shfl_up(incl, o, 64);
    if (lane >= o) incl += u;
  }
  __syncthreads();                  // the sums of an earlier call have been read
  if (lane == 63) wave_sums[wave] = incl;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const T s = wave_sums[w];
    if (w < wave) before += s;
    all += s;
  }
  total = all;
  return before + incl - v;
}

// For each of U values x: the last i in [0, n) with first[i] <= x (first ascending, first[0] <= x); among equal entries the last, so that of requests
// without rows in front of one that has some the latter is found.  The same steps for all, so that their reads are in flight together.
template <int U>
__device__ __forceinline__ void last_at_most(const int* first, int n, const int (&x)[U], int (&at)[U]) {
#pragma unroll
  for (int u = 0; u < U; ++u) at[u] = 0;
  for (int step = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0; step; step >>= 1)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int to = at[u] + step;
      if (to < n && first[min(to, n - 1)] <= x[u]) at[u] = to;
    }
}

// Position and place of row t of the new tokens, which is token t - cu[i] of request i
__device__ __forceinline__ void page_row(const int* table, const int* start, int max_pages, int page_shift, int i, int t_in_req, int t,
                                         int* row_pos, long long* slots) {
  const int pos = start[i] + t_in_req;
  row_pos[t] = pos;
  slots[t] = ((long long)table[(size_t)i * max_pages + (pos >> page_shift)] << page_shift) + (pos & ((1 << page_shift) - 1));
}

// Pages for a step.  Request i holds held[i] pages and needs ceil((start[i] + rows[i]) / page size) of them.  Its surplus goes onto the
// pool's stack, what it lacks comes off the stack, in the order of the requests and of their pages.  The k-th page given back lies k below
// the new top, so the next step takes it as its k-th: giving back what a step took restores the stack.  It also means that the k-th page given back in a step is the
// k-th taken in it: it goes straight from one table to the other, and every page moves by itself, in any order.
//
// page_sums: what the requests give back, take and bring, and where each one's begins among them.  Everything is
// checked before anything is written; a step that does not fit has no rows (cu all 0) and changes nothing.
// A small step is one block (page_tables_kernel): sums, pages, rows.  Its chain of four round trips to memory and four barriers is what bounds it.  Where rows may be many,
// a search per page and row is too much for one CU (200 prompts of 2000 tokens, 18k pages, 280k rows: 20 us), so sums, pages and rows are a launch each: page_sums_kernel,
// page_moves_kernel, page_rows_kernel.
struct PageArgs {
  int *table, *held, *stack, *n_free;
  const int *start, *rows;
  int n_req, max_pages, n_pages, page_shift, max_rows;
  int *cu, *row_pos;
  long long* slots;
  int* status;
  __device__ __forceinline__ int need(int i) const { return (start[i] + rows[i] + (1 << page_shift) - 1) >> page_shift; }
};

template <int NT> struct PageSums {
  static constexpr int NWV = NT / 64;
  int ipt, i0;                 // this thread's requests: i0 .. i0 + ipt - 1
  int before[3], total[3];     // pages given back, pages taken, rows: in front of its first request, and in all
  int top0, code, detail;
  int h0, need0, r0;           // its first request's pages held and needed, and rows: mostly the only one
  __device__ __forceinline__ int held(const PageArgs& a, int i) const { return i == i0 ? h0 : a.held[i]; }
  __device__ __forceinline__ int need(const PageArgs& a, int i) const { return i == i0 ? need0 : a.need(i); }
  __device__ __forceinline__ int rows(const PageArgs& a, int i) const { return i == i0 ? r0 : a.rows[i]; }
};

template <int NT>
__device__ __forceinline__ PageSums<NT> page_sums(const PageArgs& a) {
  constexpr int NWV = PageSums<NT>::NWV;
  __shared__ int sums_s[3][NWV];
  __shared__ float sizes_s[3][NWV];
  __shared__ int bad_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  PageSums<NT> p;
  p.ipt = (a.n_req + NT - 1) / NT;
  p.i0 = tid * p.ipt;
  const int limit = a.max_pages << a.page_shift;             // at most 2^30
  if (tid == 0) bad_s = INT_MAX;
  p.top0 = a.n_free[0];
  p.h0 = p.need0 = p.r0 = 0;
  // as integers, and as floats, which tell whether the integers have run over
  int sum[3] = {0, 0, 0}, bad = INT_MAX;
  float size[3] = {0.f, 0.f, 0.f};
  for (int i = p.i0; i < min(p.i0 + p.ipt, a.n_req); ++i) {
    const int s = a.start[i], r = a.rows[i], h = a.held[i];
    if (s < 0 || r < 0 || h < 0 || h > a.max_pages || s > limit || r > limit - s) { bad = min(bad, i); continue; }
    const int need = (s + r + (1 << a.page_shift) - 1) >> a.page_shift;
    if (i == p.i0) { p.h0 = h; p.need0 = need; p.r0 = r; }
    const int v[3] = {max(h - need, 0), max(need - h, 0), r};
#pragma unroll
    for (int k = 0; k < 3; ++k) { sum[k] += v[k]; size[k] += (float)v[k]; }
  }
  __syncthreads();
  if (bad != INT_MAX) atomicMin(&bad_s, bad);
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int incl = wave_scan(sum[k]);
    p.before[k] = incl - sum[k];
    size[k] = wave_sum(size[k]);
    if (lane == 63) { sums_s[k][wave] = incl; sizes_s[k][wave] = size[k]; }
  }
  __syncthreads();
  float all[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int incl = wave_scan(lane < NWV ? sums_s[k][lane < NWV ? lane : 0] : 0);
    p.total[k] = __builtin_amdgcn_readlane(incl, 63);
    if (wave > 0) p.before[k] += __builtin_amdgcn_readlane(incl, wave - 1);
    all[k] = wave_sum(lane < NWV ? sizes_s[k][lane < NWV ? lane : 0] : 0.f);
  }
  const bool over[3] = {all[0] >= 1.1e9f, all[1] >= 1.1e9f, all[2] >= 1.1e9f};      // 2^30 and more
  p.code = p.detail = 0;
  if (p.top0 < 0 || p.top0 > a.n_pages) { p.code = -1; p.detail = -1; }
  else if (bad_s != INT_MAX) { p.code = -1; p.detail = bad_s; }
  else if (over[2] || p.total[2] > a.max_rows || over[0] || p.total[0] > a.n_pages - p.top0) { p.code = -1; p.detail = -1; }
  else if (over[1] || p.total[1] > p.top0 + p.total[0]) { p.code = -3; p.detail = over[1] ? INT_MAX : p.total[1] - p.total[0] - p.top0; }
  return p;
}

// The pages that move, `step` threads side by side from number k0 on.  dyn: LDS, 4 n_req ints: the prefix sums of the pages given back and taken, and what leads from a
// number in either to a column of its request's table.
template <int NT, int U>
__device__ __forceinline__ void page_moves(const PageArgs& a, const PageSums<NT>& p, int* dyn, int k0, int step) {
  const int n = a.n_req, give = p.total[0], take = p.total[1], most = max(give, take), top = p.top0 + give;
  if (most == 0) return;
  int *give_s = dyn, *give_from = dyn + n, *take_s = dyn + 2 * n, *take_from = dyn + 3 * n;
  int g = p.before[0], t = p.before[1];
  for (int i = p.i0; i < min(p.i0 + p.ipt, n); ++i) {
    const int h = p.held(a, i), need = p.need(a, i);
    give_s[i] = g; give_from[i] = need - g;
    take_s[i] = t; take_from[i] = h - t;
    g += max(h - need, 0);
    t += max(need - h, 0);
  }
  __syncthreads();
  for (; k0 < most; k0 += U * step) {
    int k[U], i[U], page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = min(k0 + u * step, most - 1);
    // where it is: in the table of who gives it back, or on the stack
    if (give) {
      int kg[U];
#pragma unroll
      for (int u = 0; u < U; ++u) kg[u] = min(k[u], give - 1);
      last_at_most<U>(give_s, n, kg, i);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool back = k[u] < give;
      int* from = back ? a.table + (size_t)i[u] * a.max_pages + give_from[i[u]] + k[u] : a.stack + top - 1 - k[u];
      page[u] = *from;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + u * step < most) *(k[u] < give ? a.table + (size_t)i[u] * a.max_pages + give_from[i[u]] + k[u] : a.stack + top - 1 - k[u]) = -1;
    // where it goes
    if (take) {
      int kt[U];
#pragma unroll
      for (int u = 0; u < U; ++u) kt[u] = min(k[u], take - 1);
      last_at_most<U>(take_s, n, kt, i);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + u * step < most) *(k[u] < take ? a.table + (size_t)i[u] * a.max_pages + take_from[i[u]] + k[u] : a.stack + top - 1 - k[u]) = page[u];
  }
}

template <int NT>
__global__ void __launch_bounds__(NT) page_tables_kernel(PageArgs a) {
  extern __shared__ int page_dyn_smem[];
  const PageSums<NT> p = page_sums<NT>(a);
  const int tid = threadIdx.x, n = a.n_req;
  if (tid == 0) { a.status[0] = p.code; a.status[1] = p.detail; }
  if (p.code) {
    for (int i = tid; i <= n; i += NT) a.cu[i] = 0;
    return;
  }
  page_moves<NT, 1>(a, p, page_dyn_smem, tid, NT);
  __syncthreads();                // the search's arrays are free, and entries written
  int at = p.before[2];
  for (int i = p.i0; i < min(p.i0 + p.ipt, n); ++i) {
    page_dyn_smem[i] = at;
    a.cu[i] = at;
    at += p.rows(a, i);
    if (p.need(a, i) != p.held(a, i)) a.held[i] = p.need(a, i);
  }
  if (tid == 0) { a.cu[n] = p.total[2]; a.n_free[0] = p.top0 + p.total[0] - p.total[1]; }
  __syncthreads();
  for (int t = tid; t < p.total[2]; t += NT) {
    const int x[1] = {t};
    int i[1];
    last_at_most<1>(page_dyn_smem, n, x, i);
    page_row(a.table, a.start, a.max_pages, a.page_shift, i[0], t - page_dyn_smem[i[0]], t, a.row_pos, a.slots);
  }
}

__global__ void __launch_bounds__(1024) page_sums_kernel(PageArgs a) {
  const PageSums<1024> p = page_sums<1024>(a);
  if (threadIdx.x == 0) { a.status[0] = p.code; a.status[1] = p.detail; }
  int at = p.before[2];
  for (int i = p.i0; i < min(p.i0 + p.ipt, a.n_req); ++i) {
    a.cu[i] = p.code ? 0 : at;
    at += p.code ? 0 : p.rows(a, i);
  }
  if (threadIdx.x == 0) a.cu[a.n_req] = p.code ? 0 : p.total[2];
}

// (the sums once more in every block: nothing but the caller's arrays passes from launch to launch)
__global__ void __launch_bounds__(256) page_moves_kernel(PageArgs a) {
  extern __shared__ int page_dyn_smem[];
  const PageSums<256> p = page_sums<256>(a);
  if (p.code) return;
  page_moves<256, 2>(a, p, page_dyn_smem, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

// Positions and places: a block per 1024 rows, the requests' first rows in LDS.  The last block brings the pages held up to date.
__global__ void __launch_bounds__(256) page_rows_kernel(PageArgs a) {
  extern __shared__ int page_dyn_smem[];
  const int total = a.cu[a.n_req], base = blockIdx.x * 1024;
  if (blockIdx.x == gridDim.x - 1) {
    const PageSums<256> p = page_sums<256>(a);
    if (p.code) return;
    for (int i = p.i0; i < min(p.i0 + p.ipt, a.n_req); ++i) a.held[i] = p.need(a, i);
    if (threadIdx.x == 0) a.n_free[0] = p.top0 + p.total[0] - p.total[1];
    return;
  }
  if (base >= total) return;
  for (int i = threadIdx.x; i < a.n_req; i += 256) page_dyn_smem[i] = a.cu[i];
  __syncthreads();
  int t[4], i[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) t[u] = min(base + (int)threadIdx.x + 256 * u, total - 1);      // (beyond the last: the last one again)
  last_at_most<4>(page_dyn_smem, a.n_req, t, i);
#pragma unroll
  for (int u = 0; u < 4; ++u) page_row(a.table, a.start, a.max_pages, a.page_shift, i[u], t[u] - page_dyn_smem[i[u]], t[u], a.row_pos, a.slots);
}

// Elements of one type to the pool, four or two at a time, each rounded to nearest even once
template <int N> __device__ __forceinline__ void store_elems(float* p, const float (&x)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) p[e] = x[e];
}
template <int N> __device__ __forceinline__ void store_elems(bf16_t* p, const float (&x)[N]) {
#pragma unroll
  for (int e = 0; e < N; e += 2) *(uint32_t*)(p + e) = pack_bf16x2(x[e], x[e + 1]);
}

// The new tokens' keys - RMS norm with gain (k_gain null: none), then the rotation of the pairs (i, i + HD/2) by the angles of the token's
// position (rope_tab null: none) - and values, rounded to the pool's type and stored in their places.  16 lanes take one (row, KV head):
// its key and its value, HD/32 pairs a lane, so that a wave's loads are runs of 256 bytes and the norm's sum stays inside a DPP row.  Rows at
// and behind cu[n_req], and rows whose place or position is out of range, are not stored.
template <typename CT, int HD>
__global__ void __launch_bounds__(256) paged_append_kernel(const float* __restrict__ qkv, long ld, const int* __restrict__ cu, const int* __restrict__ row_pos,
                                                           const long long* __restrict__ slots, const CT* __restrict__ k_gain, const float2* __restrict__ rope_tab,
                                                           float eps, PagedView pv) {
  constexpr int half = HD / 2, HL = AttRow<HD>::HL;
  const int l = threadIdx.x & 15;
  const long v = (long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int t = (int)(v / pv.nkv), g = (int)(v - (long)t * pv.nkv);
  if (t >= min(pv.max_rows, cu[pv.n_req])) return;          // whole rows of 16 lanes
  const int pos = row_pos[t];
  const long long slot = slots[t];
  AttRow<HD> k, w;
  k.load(qkv + (size_t)t * ld + (size_t)(pv.nh + g) * HD, l);
  w.load(qkv + (size_t)t * ld + (size_t)(pv.nh + pv.nkv + g) * HD, l);
  if (pos < 0 || pos >= pv.limit || slot < 0 || slot >= ((long long)pv.n_pages << pv.page_shift)) return;
  float x0[HL], x1[HL], ss = 0.f;
#pragma unroll
  for (int e = 0; e < HL; ++e) { x0[e] = k.a[e]; x1[e] = k.b[e]; ss += x0[e] * x0[e] + x1[e] * x1[e]; }
  if (k_gain) {
    const float rs = rsqrtf(row16_sum(ss) / (float)HD + eps);
#pragma unroll
    for (int e = 0; e < HL; ++e) { x0[e] *= rs * Elem<CT>::to_f32(k_gain[HL * l + e]); x1[e] *= rs * Elem<CT>::to_f32(k_gain[half + HL * l + e]); }
  }
  if (rope_tab) {
    const float2* rp = rope_tab + (size_t)pos * half + HL * l;
#pragma unroll
    for (int e = 0; e < HL; ++e) {
      const float2 cs = rp[e];
      const float a = x0[e], b = x1[e];
      x0[e] = a * cs.x - b * cs.y;
      x1[e] = b * cs.x + a * cs.y;
    }
  }
  const size_t at = (size_t)(slot >> pv.page_shift) * pv.page_stride + (((size_t)g << pv.page_shift) + (size_t)(slot & ((1 << pv.page_shift) - 1))) * HD + HL * l;
  store_elems<HL>((CT*)pv.k + at, x0);
  store_elems<HL>((CT*)pv.k + at + half, x1);
#pragma unroll
  for (int e = 0; e < HL; ++e) { x0[e] = w.a[e]; x1[e] = w.b[e]; }
  store_elems<HL>((CT*)pv.v + at, x0);
  store_elems<HL>((CT*)pv.v + at + half, x1);
}

}  // namespace dmtd
