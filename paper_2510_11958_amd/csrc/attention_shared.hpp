// Attention of a step's new tokens where groups of requests start with the same pages: a system prompt, a document that many ask about.
//
// out = softmax(q k / sqrt(hd)) v over a request's keys is a sum over any partition of the keys: parts (m, l, o) = (maximum, sum of weights 2^(s - m), sum of weights x values)
// join as m = max m_i, l = sum 2^(m_i - m) l_i, o = sum 2^(m_i - m) o_i.  So the rows of all requests of a group attend to the pages that the group shares together, as the rows of one
// request that sees all of them, and each request's rows attend to what lies behind these pages for themselves; the blocks are those of the paged attention (paged_few_item,
// paged_tall_item), which find their rows through a list.  A shared key is read once per 128 query vectors (or 16, where the group has few) instead of once per request.
//
// share_plan_kernel, once a step, lays the work out for all layers: the items (a tile of rows x a range of keys), longest kind first, and what every row's parts are.  Then, per layer,
// paged_shared_mfma_kernel takes the items, whose number only the device knows, with as many blocks as the chip holds, and paged_shared_join_kernel joins the parts.
// Bound: shared keys and values once for each tile of rows, own ones once, against 4 hd x keys x query vectors operations (twice that for queries and probabilities in two parts); a vector's
// parts of 4 (hd + 2) bytes go out and come back once per range.
#pragma once
#include "attention_paged.hpp"

namespace dmtd {

constexpr int SHARE_HEADER = 16;      // ints in front of the items: sign, tall items, items, rows
// Query vectors of an entry up to which its tiles are single waves' (us a layer with 32 / 64: 16 requests of 4 vectors behind 16384 shared tokens 39 / 51, 8 of 6 behind 8192, 8-bit, 27 / 30)
constexpr int SHARE_FEW = 32;
// Items of single waves that the key ranges are chosen for: four on each CU (us a layer with 512 / 1024 / 2048: 40 requests of 2000 own tokens, 8-bit, 70 / 46 / 49, 20 of 3000, 14/2 heads of 64, 21 / 19 / 19,
// 8 behind 4096 shared tokens 19 / 21 / 21)
constexpr int SHARE_SLOTS_FEW = 1024;
// Items of blocks that the key ranges are chosen for: one on each CU, which reads as fast as it works, and two where one would have SHARE_LONG keys and more: both together do 1.3 times the work, at the
// cost of twice the parts (us a layer with one / two: 458 rows of 14/2 heads of 64 behind 10000 73 / 56, 5 chunks of 300 behind 3000 107 / 89; 64 rows of 32/8 heads behind 16384 60 / 67)
constexpr int SHARE_SLOTS_TALL = 256, SHARE_LONG = 1536;
// Shortest range of a wave with an fp32 cache, whose products weigh more (of the others: PAGED_KEYS_FEW; us with 64 / 128: 10 rows of 4/2 heads of 64, one layer and the plan, 17.6 / 20.8, 20 single tokens behind
// 500 shared ones, a layer, 12 / 15, 6 rows of 32/8 heads of 128 behind 1000 17 / 22)
constexpr int SHARE_KEYS_FP32 = 64;
constexpr int kShareMaxGroups = kPagedMaxRequests;
constexpr int SHARE_LDS_ENTRIES = 1024;      // requests, and groups, up to which a plan is worked out in LDS

// A plan in the caller's memory
struct SharePlan {
  int* head;            // SHARE_HEADER ints
  int4* items;          // two each: (req, row0, r, pos0), (kb, ke, unit, step)
  int2* list;           // [max_rows] (row, position) of the rows that see a prefix, group by group
  int4* recs;           // [max_rows][2]: unit of the row's first own part, parts, units from one to the next, 0; the same of its prefix
  int* scratch;         // what a plan of many requests is worked out in
};

struct ShareArgs {
  const int *start, *cu, *group, *pages;      // [n_req], [n_req + 1], [n_req], [n_groups]
  int n_groups, few_shift, tall_shift, few_max, few_keys;      // few_max: query vectors of an entry up to which its tiles are single waves', few_keys: the shortest range of these
  int sign;
  SharePlan plan;
};

// What a plan knows of its requests and groups: rows, keys (of a request: behind its prefix) and where its first unit, item and place in the list are
struct ShareTables {
  int *first, *n, *start, *group, *prefix, *place, *unit, *tall, *few;      // of the requests; first: [n_req + 1]
  int *g_n, *g_head, *g_keys, *g_unit, *g_list, *g_tall, *g_few;            // of the groups
  static constexpr int REQ = 9, GROUP = 7;
  static __host__ __device__ long ints(int n_req, int n_groups) { return (long)REQ * n_req + 1 + (long)GROUP * n_groups; }
  __device__ __forceinline__ ShareTables(int* at, int n_req, int n_groups) {
    int** r[REQ] = {&n, &start, &group, &prefix, &place, &unit, &tall, &few, &first};
#pragma unroll
    for (int k = 0; k < REQ; ++k) *r[k] = at + (long)k * n_req;
    int** g[GROUP] = {&g_n, &g_head, &g_keys, &g_unit, &g_list, &g_tall, &g_few};
#pragma unroll
    for (int k = 0; k < GROUP; ++k) *g[k] = at + (long)REQ * n_req + 1 + (long)k * n_groups;
  }
};

// The plan of a step, in one block.  Own entries are the requests, with the keys behind their prefix; prefix entries are the groups of two requests and more that have rows.  A request
// takes part in its group if its tokens reach beyond the prefix, and goes by itself over its whole table otherwise.  Its place among the group's rows is given out by an atomic add: where a
// row stands in its tile has no influence on its results.  All ranges of a kind have kps keys, chosen as in paged_find.
// Bound by its chain of round trips and barriers: three of the former, the tables being in LDS (57 requests: 7.0 to 7.4 us; with the tables in memory 11.8).
// LDS false: more requests or groups than that; the tables are in the plan's scratch, the groups' counts still in LDS.
template <int NT, bool LDS>
__global__ void __launch_bounds__(NT) share_plan_kernel(ShareArgs a, PagedView pv) {
  extern __shared__ int share_dyn_smem[];
  __shared__ unsigned long long total_s[3][NT / 64];
  __shared__ int scan_s[7][NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n_req = pv.n_req, n_groups = a.n_groups;
  const SharePlan& P = a.plan;
  ShareTables T(LDS ? share_dyn_smem : P.scratch, n_req, n_groups);
  if (!LDS) { T.g_n = share_dyn_smem; T.g_head = share_dyn_smem + n_groups; }
  const int ipr = (n_req + NT - 1) / NT, r0 = min(tid * ipr, n_req), r1 = min(r0 + ipr, n_req);
  const int ipg = (n_groups + NT - 1) / NT, g0 = min(tid * ipg, n_groups), g1 = min(g0 + ipg, n_groups);
  // mostly a thread's only request and group: all asked for before any is waited for
  const int i0 = min(r0, n_req - 1), end_of_all = a.cu[n_req], first0 = a.cu[i0], end0 = a.cu[i0 + 1], start0 = a.start[i0], group0 = a.group[i0], pages0 = a.pages[min(g0, n_groups - 1)];
#pragma unroll 1
  for (int g = g0; g < g1; ++g) {
    const int pages = g == g0 ? pages0 : a.pages[g];
    T.g_n[g] = 0;
    T.g_head[g] = INT_MAX;
    T.g_keys[g] = pages > 0 && pages <= pv.max_pages ? pages << pv.page_shift : 0;
  }
  bool descends = false;
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    const bool own = i == r0;
    const PagedReq q = paged_req(pv, own ? first0 : a.cu[i], own ? end0 : a.cu[i + 1], own ? start0 : a.start[i], INT_MAX, descends);
    T.first[i] = q.first;
    T.n[i] = q.n;
    T.start[i] = q.start;
    T.group[i] = own ? group0 : a.group[i];
  }
  if (__syncthreads_or(descends)) {
    if (tid == 0) { P.head[0] = a.sign; P.head[1] = P.head[2] = P.head[3] = 0; }
    return;
  }
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    const int g = T.group[i], keys = g >= 0 && g < n_groups ? T.g_keys[g] : 0;
    const bool in = T.n[i] > 0 && keys > 0 && keys <= T.start[i];
    T.prefix[i] = in ? keys : 0;
    if (in) {
      T.place[i] = atomicAdd(&T.g_n[g], T.n[i]);
      atomicMin(&T.g_head[g], i);
    }
  }
  __syncthreads();
  auto tall_of = [&](int n) { return (long)n * pv.gq > a.few_max; };
  auto rpb_of = [&](bool tall) { return tall ? pv.rpb_tall : pv.rpb_few; };
  auto tiles_of = [&](int n, bool tall) { return (int)((unsigned)(n + rpb_of(tall) - 1) / (unsigned)rpb_of(tall)); };
  // a group that is one request goes by itself
  unsigned long long sum[3] = {0, 0, 0};      // keys of the tiles of either kind, tall tiles
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    const int n = T.n[i], g = T.group[i];
    if (T.prefix[i] && T.g_n[g] == n) T.prefix[i] = 0;
    const bool tall = tall_of(n);
    const int tiles = tiles_of(n, tall);
    sum[tall] += (unsigned long long)tiles * (unsigned)(T.start[i] + n - T.prefix[i]);
    sum[2] += tall ? tiles : 0;
  }
#pragma unroll 1
  for (int g = g0; g < g1; ++g) {
    const int n = T.g_n[g], h = T.g_head[g];
    if (n == 0) continue;
    if (T.n[h] == n) { T.g_keys[g] = 0; continue; }      // (no rows of it below either)
    const bool tall = tall_of(n);
    const int tiles = tiles_of(n, tall);
    sum[tall] += (unsigned long long)tiles * (unsigned)T.g_keys[g];
    sum[2] += tall ? tiles : 0;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    sum[k] = wave_reduce(sum[k], [](unsigned long long x, unsigned long long y) { return x + y; });
    if (lane == 0) total_s[k][wave] = sum[k];
  }
  __syncthreads();
  // keys of a range of either kind: rows are at most 2^24, keys 2^30
  int kps[2];
  unsigned long long tall_tiles = 0;
  for (int w = 0; w < NT / 64; ++w) tall_tiles += total_s[2][w];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    unsigned long long all = 0;
    for (int w = 0; w < NT / 64; ++w) all += total_s[k][w];
    const int shift = k ? a.tall_shift : a.few_shift;
    unsigned long long per = (all + (1ull << shift) - 1) >> shift;
    if (k && per >= SHARE_LONG) {
      // every tile's last range may be a short one: of 2^(shift + 1) items, no more than the chip holds, those are set aside, if that leaves most of them (16 items in a second round: 66 us for 56)
      const unsigned items = (2u << shift) - (tall_tiles < (1ull << shift) ? (unsigned)tall_tiles : 0u);
      per = (all + items - 1) / items;
    }
    kps[k] = (int)min(max((unsigned long long)(k ? PAGED_KEYS_TALL : a.few_keys), (per + 63) / 64 * 64), 1ull << 30);
  }
  auto ranges_of = [&](int keys, bool tall) { return (int)((unsigned)(keys + kps[tall] - 1) / (unsigned)kps[tall]); };
  // tall and few items of the requests and of the groups, units of either, places in the list: of this thread, in front of it, and of all
  int v[7] = {0, 0, 0, 0, 0, 0, 0}, all[7];
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    const int n = T.n[i];
    if (!n) continue;
    const bool tall = tall_of(n);
    const int parts = ranges_of(T.start[i] + n - T.prefix[i], tall), count = tiles_of(n, tall) * parts;
    v[0] += tall ? count : 0;
    v[1] += tall ? 0 : count;
    v[2] += T.prefix[i] || parts > 1 ? n * parts : 0;
  }
#pragma unroll 1
  for (int g = g0; g < g1; ++g) {
    const int n = T.g_keys[g] ? T.g_n[g] : 0;
    if (!n) continue;
    const bool tall = tall_of(n);
    const int parts = ranges_of(T.g_keys[g], tall), count = tiles_of(n, tall) * parts;
    v[3] += tall ? count : 0;
    v[4] += tall ? 0 : count;
    v[5] += n * parts;
    v[6] += n;
  }
#pragma unroll
  for (int k = 0; k < 7; ++k) {
    const int incl = wave_scan(v[k]);
    if (lane == 63) scan_s[k][wave] = incl;
    v[k] = incl - v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 7; ++k) {
    all[k] = 0;
    for (int w = 0; w < NT / 64; ++w) {
      const int x = scan_s[k][w];
      v[k] += w < wave ? x : 0;
      all[k] += x;
    }
  }
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    T.tall[i] = v[0];
    T.few[i] = v[1];
    T.unit[i] = v[2];
    const int n = T.n[i];
    if (!n) continue;
    const bool tall = tall_of(n);
    const int parts = ranges_of(T.start[i] + n - T.prefix[i], tall), count = tiles_of(n, tall) * parts;
    v[0] += tall ? count : 0;
    v[1] += tall ? 0 : count;
    v[2] += T.prefix[i] || parts > 1 ? n * parts : 0;
  }
#pragma unroll 1
  for (int g = g0; g < g1; ++g) {
    T.g_tall[g] = v[3];
    T.g_few[g] = v[4];
    T.g_unit[g] = all[2] + v[5];
    T.g_list[g] = v[6];
    const int n = T.g_keys[g] ? T.g_n[g] : 0;
    if (!n) continue;
    const bool tall = tall_of(n);
    const int parts = ranges_of(T.g_keys[g], tall), count = tiles_of(n, tall) * parts;
    v[3] += tall ? count : 0;
    v[4] += tall ? 0 : count;
    v[5] += n * parts;
    v[6] += n;
  }
  const int n_rows = min(max(end_of_all, 0), pv.max_rows), n_tall = all[3] + all[0], n_items = n_tall + all[4] + all[1];
  if (tid == 0) { P.head[0] = a.sign; P.head[1] = n_tall; P.head[2] = n_items; P.head[3] = n_rows; }
  __syncthreads();
  // items: the groups' tall ones, the requests', then the few-rows ones likewise
#pragma unroll 1
  for (int y = tid; y < n_items; y += NT) {
    const bool tall = y < n_tall;
    const int in_kind = tall ? y : y - n_tall, shared_ones = tall ? all[3] : all[4], len = kps[tall], rpb = rpb_of(tall);
    const bool shared = in_kind < shared_ones;
    const int x[1] = {shared ? in_kind : in_kind - shared_ones};
    int at[1];
    const int* first = shared ? (tall ? T.g_tall : T.g_few) : (tall ? T.tall : T.few);
    last_at_most<1>(first, shared ? n_groups : n_req, x, at);
    const int i = at[0], rel = x[0] - first[i], n = shared ? T.g_n[i] : T.n[i], keys = shared ? T.g_keys[i] : T.start[i] + n - T.prefix[i];
    const int parts = ranges_of(keys, tall), tile = (int)((unsigned)rel / (unsigned)parts), k = rel - tile * parts, row0 = tile * rpb, r = min(rpb, n - row0);
    int4 u, w;
    if (shared) {
      u = make_int4(T.g_head[i], T.g_list[i] + row0, r, keys - 1);
      w = make_int4(k * len, min(keys, k * len + len), T.g_unit[i] + k * n + row0, 0);
    } else {
      const int front = T.prefix[i], pos0 = T.start[i] + row0, end = pos0 + r;
      const bool whole = front == 0 && end <= len;
      u = make_int4(i, T.first[i] + row0, r, pos0);
      w = make_int4(front + k * len, min(end, front + k * len + len), whole ? -1 : T.unit[i] + k * n + row0, 1);
    }
    P.items[2 * y] = u;
    P.items[2 * y + 1] = w;
  }
#pragma unroll 1
  for (int t = tid; t < n_rows; t += NT) {
    const int x[1] = {t};
    int at[1];
    last_at_most<1>(T.first, n_req, x, at);
    const int i = at[0], j = t - T.first[i], n = T.n[i];
    int4 u = make_int4(0, 0, 0, 0), w = u;
    if (j >= 0 && j < n) {
      const bool tall = tall_of(n);
      const int rpb = rpb_of(tall), front = T.prefix[i], seen = T.start[i] + min((int)((unsigned)j / (unsigned)rpb) * rpb + rpb, n) - front, parts = ranges_of(seen, tall);
      if (front || parts > 1) u = make_int4(T.unit[i] + j, parts, n, 0);
      if (front) {
        const int g = T.group[i], place = T.place[i] + j;
        P.list[T.g_list[g] + place] = make_int2(t, T.start[i] + j);
        w = make_int4(T.g_unit[g] + place, ranges_of(front, tall_of(T.g_n[g])), T.g_n[g], 0);
      }
    }
    P.recs[2 * t] = u;
    P.recs[2 * t + 1] = w;
  }
}

// The items of a plan, head by head, over a grid of blocks that the chip holds.  Tall ones are a block's: with 8 KV heads (or a multiple) block b's are of one head, whose keys stay in
// the L2 of the block's die.  Then the others, a wave's each: those of the blocks with fewer tall ones come first.
// The first item is asked for beside the plan's numbers, which say whether it is one.  most: items that the plan has room for.
template <typename CT, int HD, bool TALL>
__global__ void __launch_bounds__(256, 2) paged_shared_mfma_kernel(SharePlan plan, int sign, int most, const float* __restrict__ qkv, long ld, const typename PagedWide<CT>::type* __restrict__ q_gain,
                                                                   const float2* __restrict__ rope_tab, float eps, PagedOut po, PagedView pv, SharedParts sp) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grid = gridDim.x;
  auto item_at = [&](int item) {
    const int4 u = plan.items[2 * item], v = plan.items[2 * item + 1];
    return SharedItem{__builtin_amdgcn_readfirstlane(u.x), __builtin_amdgcn_readfirstlane(u.y), __builtin_amdgcn_readfirstlane(u.z), __builtin_amdgcn_readfirstlane(u.w),
                      __builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z), __builtin_amdgcn_readfirstlane(v.w)};
  };
  const int4 head = *(const int4*)plan.head;
  SharedItem it = item_at(min((int)((unsigned)(TALL ? blockIdx.x : wave * grid + blockIdx.x) / (unsigned)pv.nkv), most - 1));
  if (__builtin_amdgcn_readfirstlane(head.x) != sign) return;
  const int n_tall = TALL ? __builtin_amdgcn_readfirstlane(head.y) : 0, all_tall = n_tall * pv.nkv, all_few = __builtin_amdgcn_readfirstlane(head.z) * pv.nkv - all_tall;
  // the lane's number and what follows from it are worked out anew for each item: kept through the loop they would be spilled
  auto lane_now = [&] {
    unsigned zero = 0;
    asm volatile("" : "+v"(zero));
    return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
  };
  if constexpr (TALL) {
    for (int y = blockIdx.x; y < all_tall; y += grid) {
      const int item = (int)((unsigned)y / (unsigned)pv.nkv), g = y - item * pv.nkv;
      if (y != (int)blockIdx.x) it = item_at(item);
      if (it.kb < it.ke) paged_tall_item<CT, HD, false, true>(it, g, 64 * wave + lane_now(), qkv, ld, q_gain, rope_tab, eps, po, pv, PagedWork{}, sp);      // (or keys that the tile's rows do not reach)
      __syncthreads();                          // the item's LDS is free
    }
  }
  const int more = all_tall % grid, fewer = grid - more, rank = (int)blockIdx.x >= more ? blockIdx.x - more : fewer + blockIdx.x;
  for (int y = rank < fewer ? wave * fewer + rank : 4 * fewer + wave * more + rank - fewer; y < all_few; y += 4 * grid) {
    const int item = (int)((unsigned)y / (unsigned)pv.nkv), g = y - item * pv.nkv;
    if (TALL || y >= 4 * grid) it = item_at(n_tall + item);
    if (it.kb < it.ke) paged_few_item<CT, HD, false, true>(it, g, lane_now(), wave, qkv, ld, q_gain, rope_tab, eps, po, pv, PagedWork{}, sp);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // the item's LDS is free
    __builtin_amdgcn_wave_barrier();
  }
}

// A row's parts joined, first the prefix's, then its own, each in the order of the keys: 4 dims of a head a thread, and as many threads as a wave has for it share the parts.  Rows with one part have been written.
template <typename GT, int HD>
__global__ void __launch_bounds__(256) paged_shared_join_kernel(SharePlan plan, int sign, PagedOut po, PagedView pv, SharedParts sp) {
  constexpr int T4 = HD / 4, SHARE = 64 / T4, U = 4;      // U: parts of a thread in flight
  const int turn = (threadIdx.x & 63) / T4, d = (threadIdx.x % T4) * 4;
  const long first = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  // the first row's parts are asked for beside the plan's numbers
  const int4 numbers = *(const int4*)plan.head;
  const int t0 = min((int)(first / pv.nh), pv.max_rows - 1);
  int4 own = plan.recs[2 * t0], front = plan.recs[2 * t0 + 1];
  if (numbers.x != sign) return;
  const long total = (long)numbers.w * pv.nh;
  for (long e = first; e < total; e += (long)gridDim.x * 4) {
    const int t = (int)(e / pv.nh), head = (int)(e - (long)t * pv.nh);
    if (e != first) { own = plan.recs[2 * t]; front = plan.recs[2 * t + 1]; }
    if (own.y == 0) continue;
    // part k of the row: of the prefix, then its own
    const int n = front.y + own.y;
    auto unit = [&](int k) { return k < front.y ? front.x + k * front.z : own.x + (k - front.y) * own.z; };
    PagedSum sum;
    for (int k0 = turn; k0 < n; k0 += U * SHARE) {
      float2 w[U];
      f32x4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 + u * SHARE < n) {
          const int at = unit(k0 + u * SHARE);
          w[u] = *(const float2*)sp.weights(at, pv.nh, head, HD);
          x[u] = *(const f32x4*)(sp.sums(at, head, HD) + d);
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 + u * SHARE < n) sum.add(w[u].x, w[u].y, x[u]);
    }
#pragma unroll
    for (int o = T4; o < 64; o *= 2)
      sum.add(__shfl_xor(sum.m, o, 64), __shfl_xor(sum.l, o, 64), f32x4{__shfl_xor(sum.o.x, o, 64), __shfl_xor(sum.o.y, o, 64), __shfl_xor(sum.o.z, o, 64), __shfl_xor(sum.o.w, o, 64)});
    if (turn == 0) paged_store4<GT, false>(po, t, head * HD + d, sum.result());
  }
}

}  // namespace dmtd
