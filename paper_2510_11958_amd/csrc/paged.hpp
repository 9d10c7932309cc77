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
  if (NT == 64) {
    total = __shfl(incl, 63, 64);
    return incl - v;
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
// the new top, so the next step takes it as its k-th: giving back what a step took restores the stack.
// One block, whose threads hold up to RPT requests each: three prefix sums, and a search in one of them for each page that moves and for
// each row.  Everything is checked before anything is written; a step that does not fit has no rows (cu all 0) and changes nothing.
// Bound by latency: a chain of four round trips to memory (lengths; pages off the stack; their entries read for the rows' places; the last stores) and five
// barriers.  us in a stream of calls: one request 2.9; 256, of which 19 grow by a page 6.2 with 1024 threads, three sums one after the other and
// lengths read again, 22 for 200 prompts of 2000 tokens; as it stands see below.
constexpr int PAGE_RPT = kPagedMaxRequests / 1024;
template <int NT>
__global__ void __launch_bounds__(NT) page_tables_kernel(int* __restrict__ table, int* __restrict__ held, int* __restrict__ stack, int* __restrict__ n_free,
                                                         const int* __restrict__ start, const int* __restrict__ rows, int n_req, int max_pages, int n_pages,
                                                         int page_shift, int max_rows, int* __restrict__ cu, int* __restrict__ row_pos,
                                                         long long* __restrict__ slots /* null: page_rows_kernel follows */, int* __restrict__ status) {
  constexpr int NWV = NT / 64, RPT = NT == 1024 ? PAGE_RPT : 1;
  __shared__ int first_s[NT * RPT];
  __shared__ int sums_s[3][NWV];
  __shared__ float sizes_s[3][NWV];
  __shared__ int bad_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ipt = (n_req + NT - 1) / NT, i0 = tid * ipt;
  const int limit = max_pages << page_shift;             // at most 2^30
  if (tid == 0) bad_s = INT_MAX;
  const int top0 = n_free[0];
  int s[RPT], r[RPT], h[RPT], need[RPT];
#pragma unroll
  for (int j = 0; j < RPT; ++j) {
    const bool on = j < ipt && i0 + j < n_req;
    s[j] = on ? start[i0 + j] : 0;
    r[j] = on ? rows[i0 + j] : 0;
    h[j] = on ? held[i0 + j] : 0;
  }
  __syncthreads();
  // pages given back, pages taken, rows: as integers, and as floats, which tell whether the integers have run over
  int sum[3] = {0, 0, 0};
  float size[3] = {0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < RPT; ++j) {
    const bool fits = s[j] >= 0 && r[j] >= 0 && h[j] >= 0 && h[j] <= max_pages && s[j] <= limit && r[j] <= limit - s[j];
    if (!fits) atomicMin(&bad_s, i0 + j);
    need[j] = fits ? (s[j] + r[j] + (1 << page_shift) - 1) >> page_shift : 0;
    const int v[3] = {max(h[j] - need[j], 0), max(need[j] - h[j], 0), r[j]};
#pragma unroll
    for (int k = 0; k < 3; ++k) { sum[k] += fits ? v[k] : 0; size[k] += fits ? (float)v[k] : 0.f; }
  }
  int before[3], total[3] = {0, 0, 0};
  float all[3] = {0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int incl = wave_scan(sum[k]);
    before[k] = incl - sum[k];
    size[k] = wave_sum(size[k]);
    if (lane == 63) { sums_s[k][wave] = incl; sizes_s[k][wave] = size[k]; }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int w = 0; w < NWV; ++w) {
      const int u = sums_s[k][w];
      if (w < wave) before[k] += u;
      total[k] += u;
      all[k] += sizes_s[k][w];
    }
  const bool over[3] = {all[0] >= 1.1e9f, all[1] >= 1.1e9f, all[2] >= 1.1e9f};      // 2^30 and more
  int code = 0, detail = 0;
  if (top0 < 0 || top0 > n_pages) { code = -1; detail = -1; }
  else if (bad_s != INT_MAX) { code = -1; detail = bad_s; }
  else if (over[2] || total[2] > max_rows || over[0] || total[0] > n_pages - top0) { code = -1; detail = -1; }
  else if (over[1] || total[1] > top0 + total[0]) { code = -3; detail = over[1] ? INT_MAX : total[1] - total[0] - top0; }
  if (tid == 0) { status[0] = code; status[1] = detail; }
  if (code) {
    for (int i = tid; i <= n_req; i += NT) cu[i] = 0;
    return;
  }
  const int give = total[0], take = total[1], n_rows = total[2], top = top0 + give;
  // a prefix sum into LDS, for searches in it
  auto lay_out = [&](int k) {
    int at = before[k];
#pragma unroll
    for (int j = 0; j < RPT; ++j)
      if (j < ipt && i0 + j < n_req) {
        first_s[i0 + j] = at;
        at += k == 0 ? max(h[j] - need[j], 0) : k == 1 ? max(need[j] - h[j], 0) : r[j];
      }
    __syncthreads();
  };
  constexpr int U = NT == 1024 ? 4 : 1;       // pages and rows in flight per thread
  if (give) {
    lay_out(0);
    for (int k0 = tid; k0 < give; k0 += U * NT) {
      int k[U], i[U], page[U];
      int* entry[U];
#pragma unroll
      for (int u = 0; u < U; ++u) k[u] = min(k0 + u * NT, give - 1);
      last_at_most<U>(first_s, n_req, k, i);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        entry[u] = table + (size_t)i[u] * max_pages + ((start[i[u]] + rows[i[u]] + (1 << page_shift) - 1) >> page_shift) + k[u] - first_s[i[u]];
        page[u] = *entry[u];
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 + u * NT < give) { stack[top - 1 - k[u]] = page[u]; *entry[u] = -1; }
    }
    __syncthreads();                // the stack is whole before pages come off it, the search's array free again
  }
  if (take) {
    lay_out(1);
    for (int k0 = tid; k0 < take; k0 += U * NT) {
      int k[U], i[U], page[U];
      int* entry[U];
#pragma unroll
      for (int u = 0; u < U; ++u) { k[u] = min(k0 + u * NT, take - 1); page[u] = stack[top - 1 - k[u]]; }
      last_at_most<U>(first_s, n_req, k, i);
#pragma unroll
      for (int u = 0; u < U; ++u) entry[u] = table + (size_t)i[u] * max_pages + held[i[u]] + k[u] - first_s[i[u]];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 + u * NT < take) { *entry[u] = page[u]; stack[top - 1 - k[u]] = -1; }
    }
    __syncthreads();                // held is read above; entries are read below
  }
  lay_out(2);
#pragma unroll
  for (int j = 0; j < RPT; ++j)
    if (j < ipt && i0 + j < n_req) {
      cu[i0 + j] = first_s[i0 + j];
      if (need[j] != h[j]) held[i0 + j] = need[j];
    }
  if (tid == 0) { cu[n_req] = n_rows; n_free[0] = top - take; }
  if (!slots) return;
  for (int t = tid; t < n_rows; t += NT) {
    const int x[1] = {t};
    int i[1];
    last_at_most<1>(first_s, n_req, x, i);
    page_row(table, start, max_pages, page_shift, i[0], t - first_s[i[0]], t, row_pos, slots);
  }
}

// Positions and places of the rows where they are many: a block per 1024 rows, the requests' first rows in LDS
__global__ void __launch_bounds__(256) page_rows_kernel(const int* __restrict__ table, const int* __restrict__ start, int n_req, int max_pages, int page_shift,
                                                        const int* __restrict__ cu, int* __restrict__ row_pos, long long* __restrict__ slots) {
  __shared__ int first_s[kPagedMaxRequests];
  const int total = cu[n_req], base = blockIdx.x * 1024;
  if (base >= total) return;
  for (int i = threadIdx.x; i < n_req; i += 256) first_s[i] = cu[i];
  __syncthreads();
  int t[4], i[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) t[u] = min(base + (int)threadIdx.x + 256 * u, total - 1);      // (beyond the last: the last one again)
  last_at_most<4>(first_s, n_req, t, i);
#pragma unroll
  for (int u = 0; u < 4; ++u) page_row(table, start, max_pages, page_shift, i[u], t[u] - first_s[i[u]], t[u], row_pos, slots);
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
