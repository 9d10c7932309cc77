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
constexpr int kShareMaxRequests = kPagedMaxRequests, kShareMaxGroups = kPagedMaxRequests;

// A plan in the caller's memory
struct SharePlan {
  int* head;            // SHARE_HEADER ints
  int4* items;          // two each: (req, row0, r, pos0), (kb, ke, unit, step)
  int2* list;           // [max_rows] (row, position) of the step's rows, then [max_rows] of the rows that see a prefix, group by group
  int4* recs;           // [max_rows][2]: unit of the row's first own part, parts, units from one to the next, 0; the same of its prefix
  int4* reqs;           // [n_req]: tokens of the prefix, its place among the group's rows, first own unit, 0
  int4* groups;         // [n_groups]: rows, a request of the group, first unit, first place in the list
};

struct ShareArgs {
  const int *start, *cu, *group, *pages;      // [n_req], [n_req + 1], [n_req], [n_groups]
  int n_groups, few_shift, tall_shift, few_max;      // query vectors of an entry up to which it goes to the few-rows blocks
  int sign;
  SharePlan plan;
};

// What the ranges of an entry (the rows of a request, or of a group) come to
struct ShareEntry { int rows, keys, rpb, kps; bool tall; };

// The plan of a step, in one block.  Own entries are the requests, with the keys behind their prefix; prefix entries are the groups of two requests and more that have rows.  A request
// takes part in its group if its tokens reach beyond the prefix, and goes by itself over its whole table otherwise.  Its place among the group's rows is given out by an atomic add: where a
// row stands in its tile has no influence on its results.  All ranges of a kind have kps keys, chosen as in paged_find.
// A chain of round trips to memory and barriers is what bounds it.
template <int NT>
__global__ void __launch_bounds__(NT) share_plan_kernel(ShareArgs a, PagedView pv) {
  extern __shared__ int share_dyn_smem[];
  __shared__ long long sums_s[NT / 64];
  const int tid = threadIdx.x, n_req = pv.n_req, n_groups = a.n_groups, longest = max(n_req, n_groups);
  int *first_s = share_dyn_smem, *head_s = share_dyn_smem + longest;      // rows of the groups and a request of each; later an entry's first item or row
  const SharePlan& P = a.plan;
  for (int g = tid; g < n_groups; g += NT) { first_s[g] = 0; head_s[g] = INT_MAX; }
  __syncthreads();
  const int ipr = (n_req + NT - 1) / NT, r0 = min(tid * ipr, n_req), r1 = min(r0 + ipr, n_req);
  const int ipg = (n_groups + NT - 1) / NT, g0 = min(tid * ipg, n_groups), g1 = min(g0 + ipg, n_groups);
  bool descends = false;
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    const PagedReq q = paged_req(pv, a.cu, a.start, INT_MAX, i, descends);
    const int g = a.group[i], pages = g >= 0 && g < n_groups ? a.pages[g] : 0;
    int prefix = 0, place = 0;
    if (q.n > 0 && pages > 0 && pages <= pv.max_pages && (pages << pv.page_shift) <= q.start) {
      prefix = pages << pv.page_shift;
      place = atomicAdd(&first_s[g], q.n);
      atomicMin(&head_s[g], i);
    }
    P.reqs[i] = make_int4(prefix, place, 0, 0);
  }
  if (__syncthreads_or(descends)) {
    if (tid == 0) { P.head[0] = a.sign; P.head[1] = P.head[2] = P.head[3] = 0; }
    return;
  }
  auto rows_of_group = [&](int g) {      // 0 where the group is one request: that one goes by itself
    const int n = first_s[g], h = head_s[g];
    return n > 0 && a.cu[h + 1] - a.cu[h] < n ? n : 0;
  };
  auto own = [&](int i, PagedReq& q, int& prefix) {
    bool d = false;
    q = paged_req(pv, a.cu, a.start, INT_MAX, i, d);
    prefix = P.reqs[i].x;
    if (prefix && rows_of_group(a.group[i]) == 0) prefix = 0;
    const bool tall = q.n * pv.gq > a.few_max;
    return ShareEntry{q.n, q.start + q.n - prefix, tall ? pv.rpb_tall : pv.rpb_few, 0, tall};
  };
  auto shared = [&](int g) {
    const int n = rows_of_group(g);
    const bool tall = (long)n * pv.gq > a.few_max;
    return ShareEntry{n, n ? a.pages[g] << pv.page_shift : 0, tall ? pv.rpb_tall : pv.rpb_few, 0, tall};
  };
  // keys of a range of either kind: rows are at most 2^24, keys 2^30
  long long mine[2] = {0, 0}, total[2];
  PagedReq q;
  int prefix;
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    const ShareEntry e = own(i, q, prefix);
    if (e.rows) mine[e.tall] += (long long)((e.rows + e.rpb - 1) / e.rpb) * e.keys;
  }
#pragma unroll 1
  for (int g = g0; g < g1; ++g) {
    const ShareEntry e = shared(g);
    mine[e.tall] += (long long)((e.rows + e.rpb - 1) / e.rpb) * e.keys;
  }
  for (int k = 0; k < 2; ++k) (void)block_scan<NT>(mine[k], sums_s, total[k]);
  auto keys_of = [&](long long t, int shift, int least) {
    const long long per = (t + (1ll << shift) - 1) >> shift;
    return (int)min(max((long long)least, (per + 63) / 64 * 64), 1ll << 30);
  };
  const int kps[2] = {keys_of(total[0], a.few_shift, PAGED_KEYS_FEW), keys_of(total[1], a.tall_shift, PAGED_KEYS_TALL)};
  auto ranges = [&](const ShareEntry& e) { return (int)((unsigned)(e.keys + kps[e.tall] - 1) / (unsigned)kps[e.tall]); };
  auto tiles = [&](const ShareEntry& e) { return (int)((unsigned)(e.rows + e.rpb - 1) / (unsigned)e.rpb); };
  // items of either kind (tall ones in the upper half), units and places in the list, in front of each thread's entries
  long long items_own = 0, items_shared = 0, units_own = 0, units_shared = 0;      // (units_shared: places from bit 36 on)
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    const ShareEntry e = own(i, q, prefix);
    if (!e.rows) continue;
    const int n = ranges(e);
    items_own += (long long)(tiles(e) * n) << (e.tall ? 32 : 0);
    units_own += prefix || n > 1 ? (long long)e.rows * n : 0;
  }
#pragma unroll 1
  for (int g = g0; g < g1; ++g) {
    const ShareEntry e = shared(g);
    if (!e.rows) continue;
    const int n = ranges(e);
    items_shared += (long long)(tiles(e) * n) << (e.tall ? 32 : 0);
    units_shared += ((long long)e.rows << 36) + (long long)e.rows * n;
  }
  long long all_own, all_shared, all_units, none;
  const long long at_own = block_scan<NT>(items_own, sums_s, all_own), at_shared = block_scan<NT>(items_shared, sums_s, all_shared);
  long long unit_own = block_scan<NT>(units_own, sums_s, all_units), unit_shared = block_scan<NT>(units_shared, sums_s, none);
  const long long low = (1ll << 36) - 1;
#pragma unroll 1
  for (int i = r0; i < r1; ++i) {
    const ShareEntry e = own(i, q, prefix);
    const int n = e.rows ? ranges(e) : 0;
    P.reqs[i] = make_int4(prefix, P.reqs[i].y, (int)unit_own, 0);
    unit_own += prefix || n > 1 ? (long long)e.rows * n : 0;
  }
#pragma unroll 1
  for (int g = g0; g < g1; ++g) {
    const ShareEntry e = shared(g);
    P.groups[g] = make_int4(e.rows, head_s[g], (int)(all_units + (unit_shared & low)), (int)(unit_shared >> 36));
    if (e.rows) unit_shared += ((long long)e.rows << 36) + (long long)e.rows * ranges(e);
  }
  const int n_rows = min(max(a.cu[n_req], 0), pv.max_rows);
  const int tall_shared = (int)(all_shared >> 32), tall_own = (int)(all_own >> 32), few_shared = (int)(all_shared & 0xFFFFFFFF), few_own = (int)(all_own & 0xFFFFFFFF);
  if (tid == 0) { P.head[0] = a.sign; P.head[1] = tall_shared + tall_own; P.head[2] = tall_shared + tall_own + few_shared + few_own; P.head[3] = n_rows; }
  __syncthreads();          // the groups' rows are in P.groups now; the requests' and groups' records are written
  // items, section by section: an entry's first item in LDS, then an item a thread
  int base = 0;
#pragma unroll 1
  for (int sec = 0; sec < 4; ++sec) {
    const bool tall = sec < 2, is_shared = (sec & 1) == 0;
    const int count = sec == 0 ? tall_shared : sec == 1 ? tall_own : sec == 2 ? few_shared : few_own;
    if (count == 0) continue;
    auto of = [&](int i, int& pre) {
      if (is_shared) {
        const int n = P.groups[i].x;
        const bool t = (long)n * pv.gq > a.few_max;
        pre = 0;
        return ShareEntry{n, n ? a.pages[i] << pv.page_shift : 0, t ? pv.rpb_tall : pv.rpb_few, 0, t};
      }
      bool d = false;
      q = paged_req(pv, a.cu, a.start, INT_MAX, i, d);
      pre = P.reqs[i].x;
      const bool t = q.n * pv.gq > a.few_max;
      return ShareEntry{q.n, q.start + q.n - pre, t ? pv.rpb_tall : pv.rpb_few, 0, t};
    };
    __syncthreads();        // the section before has been searched
    const long long from = is_shared ? at_shared : at_own;
    int at = tall ? (int)(from >> 32) : (int)(from & 0xFFFFFFFF);
    for (int i = is_shared ? g0 : r0; i < (is_shared ? g1 : r1); ++i) {
      int pre;
      const ShareEntry e = of(i, pre);
      first_s[i] = at;
      if (e.rows && e.tall == tall) at += tiles(e) * ranges(e);
    }
    __syncthreads();
#pragma unroll 1
    for (int y = tid; y < count; y += NT) {
      const int x[1] = {y};
      int i[1], pre;
      last_at_most<1>(first_s, is_shared ? n_groups : n_req, x, i);
      const ShareEntry e = of(i[0], pre);
      const int n = ranges(e), rel = y - first_s[i[0]], tile = (int)((unsigned)rel / (unsigned)n), k = rel - tile * n, row0 = tile * e.rpb, r = min(e.rpb, e.rows - row0), len = kps[tall];
      int4 u, v;
      if (is_shared) {
        const int4 g = P.groups[i[0]];
        u = make_int4(g.y, pv.max_rows + g.w + row0, r, e.keys - 1);
        v = make_int4(k * len, min(e.keys, k * len + len), g.z + k * e.rows + row0, 0);
      } else {
        const int pos0 = q.start + row0, end = pos0 + r;
        const bool whole = pre == 0 && end <= len;
        u = make_int4(i[0], q.first + row0, r, pos0);
        v = make_int4(pre + k * len, min(end, pre + k * len + len), whole ? -1 : P.reqs[i[0]].z + k * e.rows + row0, 1);
      }
      P.items[2 * (base + y)] = u;
      P.items[2 * (base + y) + 1] = v;
    }
    base += count;
  }
  // rows
  __syncthreads();
  for (int i = tid; i < n_req; i += NT) first_s[i] = a.cu[i];
  __syncthreads();
#pragma unroll 1
  for (int t = tid; t < n_rows; t += NT) {
    const int x[1] = {t};
    int i[1];
    last_at_most<1>(first_s, n_req, x, i);
    bool d = false;
    q = paged_req(pv, a.cu, a.start, INT_MAX, i[0], d);
    const int j = t - q.first;
    int4 u = make_int4(0, 0, 0, 0), v = u;
    if (j >= 0 && j < q.n) {
      const int4 rec = P.reqs[i[0]];
      const bool tall = q.n * pv.gq > a.few_max;
      const int rpb = tall ? pv.rpb_tall : pv.rpb_few, end = q.start + min(j / rpb * rpb + rpb, q.n) - rec.x, n = (int)((unsigned)(end + kps[tall] - 1) / (unsigned)kps[tall]);
      P.list[t] = make_int2(t, q.start + j);
      if (rec.x || n > 1) u = make_int4(rec.z + j, n, q.n, 0);
      if (rec.x) {
        const int4 g = P.groups[a.group[i[0]]];
        const int len = kps[(long)g.x * pv.gq > a.few_max], place = rec.y + j;
        P.list[pv.max_rows + g.w + place] = make_int2(t, q.start + j);
        v = make_int4(g.z + place, (int)((unsigned)(rec.x + len - 1) / (unsigned)len), g.x, 0);
      }
    }
    P.recs[2 * t] = u;
    P.recs[2 * t + 1] = v;
  }
}

// The items of a plan, head by head, over a grid that the chip holds.  With 8 KV heads (or a multiple) a block's heads are those of its die, and a head's keys pass one L2.
template <typename CT, int HD, bool TALL>
__global__ void __launch_bounds__(256, !TALL && sizeof(CT) == 2 ? 3 : 2) paged_shared_mfma_kernel(SharePlan plan, int sign, const float* __restrict__ qkv, long ld,
                                                                                             const typename PagedWide<CT>::type* __restrict__ q_gain, const float2* __restrict__ rope_tab,
                                                                                             float eps, PagedOut po, PagedView pv, SharedParts sp) {
  if (plan.head[0] != sign) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_tall = TALL ? plan.head[1] : 0, total = plan.head[2] * pv.nkv;
  for (int y = blockIdx.x; y < total; y += gridDim.x) {
    const int item = (int)((unsigned)y / (unsigned)pv.nkv), g = y - item * pv.nkv;
    const int4 u = plan.items[2 * item], v = plan.items[2 * item + 1];
    const SharedItem it{__builtin_amdgcn_readfirstlane(u.x), __builtin_amdgcn_readfirstlane(u.y), __builtin_amdgcn_readfirstlane(u.z), __builtin_amdgcn_readfirstlane(u.w),
                        __builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z), __builtin_amdgcn_readfirstlane(v.w)};
    if (it.kb >= it.ke) continue;             // keys that the tile's rows do not reach
    // the thread's number and what follows from it are worked out anew for each item: kept through the loop they would be spilled
    unsigned zero = 0;
    asm volatile("" : "+v"(zero));
    const int tid = 64 * wave + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
    if constexpr (TALL) {
      if (item < n_tall) paged_tall_item<CT, HD, false, true>(it, g, tid, qkv, ld, q_gain, rope_tab, eps, po, pv, PagedWork{}, sp);
      else paged_few_item<CT, HD, false, true>(it, g, tid, qkv, ld, q_gain, rope_tab, eps, po, pv, PagedWork{}, sp);
    } else {
      paged_few_item<CT, HD, false, true>(it, g, tid, qkv, ld, q_gain, rope_tab, eps, po, pv, PagedWork{}, sp);
    }
    __syncthreads();                          // the item's LDS is free
  }
}

// A row's parts joined, first the prefix's, then its own, each in the order of the keys: 4 dims of a head a thread.  Rows with one part have been written.
template <typename GT, int HD>
__global__ void __launch_bounds__(256) paged_shared_join_kernel(SharePlan plan, int sign, PagedOut po, PagedView pv, SharedParts sp) {
  if (plan.head[0] != sign) return;
  constexpr int T4 = HD / 4;
  const int n_rows = plan.head[3];
  const unsigned per_row = (unsigned)pv.nh * T4;
  const long total = (long)n_rows * per_row;
  for (long e = (long)blockIdx.x * 256 + threadIdx.x; e < total; e += (long)gridDim.x * 256) {
    const int t = (int)(e / per_row), c = (int)(e - (long)t * per_row), head = c / T4, d = (c % T4) * 4;
    const int4 u = plan.recs[2 * t], v = plan.recs[2 * t + 1];
    if (u.y == 0) continue;
    PagedSum sum;
    if (v.y) sum.add_ranges<false>(sp.weights(v.x, pv.nh, head, HD), sp.sums(v.x, head, HD) + d, (size_t)v.z * sp.unit_floats, 0, v.y, 1);
    sum.add_ranges<false>(sp.weights(u.x, pv.nh, head, HD), sp.sums(u.x, head, HD) + d, (size_t)u.z * sp.unit_floats, 0, u.y, 1);
    paged_store4<GT, false>(po, t, head * HD + d, sum.result());
  }
}

}  // namespace dmtd
