// Attention of a step's new tokens over the paged cache of their requests (paged.hpp).  The new tokens' own keys and values are in the cache
// already (paged_append_kernel); row t of request i, at position start[i] + t, sees the request's keys 0 .. start[i] + t.
//
// Two kinds of blocks for bf16 caches.  paged_attention_few takes the requests with few query vectors per KV head (rows x query heads that share it, up to
// PAGED_FEW): blocks of 16 vectors, which read keys and values straight from the pages at the rate of the memory.  paged_attention_tall takes the
// others: blocks of 128 vectors, whose keys and values pass through LDS, bound by the matrix cores.  A step that may have both kinds is one launch of both.
// A block serves one KV head, one group of a request's rows and one range of its keys.  The ranges are found by every block itself from the
// requests' lengths (paged_find): all of one length, such that the blocks fill the chip about once, whatever the lengths are.  Where a group has several
// ranges, their partial results go through the workspace and are joined in the order of the ranges: of few vectors by the block that ends
// last, without a second launch, of many by paged_attention_merge_kernel.
#pragma once
#include "paged.hpp"
#include "gemm_wide.hpp"

namespace dmtd {

// bf16 parts in which a probability of a bf16 cache enters its products.  Rows of bf16: two, 16 of its 24 bits, twice what the output keeps (2048 rows behind 6144, 32/8 heads of 128:
// 438 us, with three 516; 0.0017 off 64 bits with either, the output's rounding).  The planes that the projections read keep 16 bits: three, which add up to all 24, as
// in the attention of the other calls (attention_mfma.hpp, attention_prefill.hpp); values that cancel would show the roundings of two.
// 8-bit caches: two as well, although a value may have been off by 2^-4 when it was stored: what is stored is what the caller has, and a part of 8 bits would add an error of the size of the
// output's own rounding (2048 rows behind 6144, 32/8 heads of 128: two parts 456 us and 0.0017 off 64 bits on the stored values, one part 377 and 0.0023).
template <bool PLANES> constexpr int PAGED_PARTS = PLANES ? 3 : 2;

// A pair of probabilities in three bf16 parts: the leading 8 bits, the next 8, the rest
__device__ __forceinline__ void paged_split3(float a, float b, uint32_t& h, uint32_t& m, uint32_t& l) {
  const float a1 = a - __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), b1 = b - __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
  const float a2 = a1 - __uint_as_float(__float_as_uint(a1) & 0xFFFF0000u), b2 = b1 - __uint_as_float(__float_as_uint(b1) & 0xFFFF0000u);
  h = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  m = __builtin_amdgcn_perm(__float_as_uint(b1), __float_as_uint(a1), 0x07060302u);
  l = __builtin_amdgcn_perm(__float_as_uint(b2), __float_as_uint(a2), 0x07060302u);
}

// Blocks that the key ranges are chosen for.  bf16, few rows: one of four waves on each CU reads as fast as more do, and shorter ranges cost more joins (us, 32/8 heads of 128,
// 256 / 512 / 1024 blocks: 3 rows of 8 requests behind 16384 84 / 85 / 95, one row behind 16384 19 / 22 / 27, 4 rows of 32 behind 1024 27 / 31 / 36).  fp32, whose
// products weigh more: 512 (16/8 heads, 200 rows behind 1000 55 / 40 / 44).  Tall: half of the blocks that the chip holds (64 rows behind 4096 27, with 512 33).
constexpr int PAGED_SLOTS_FEW = 256, PAGED_SLOTS_FP32 = 512, PAGED_SLOTS_TALL = 256;
constexpr int PAGED_RESIDENT_TALL = 512;                           // blocks of the tall kernel that the chip holds
constexpr int PAGED_WAVES = 4;                                     // waves of a block of the few-rows kernel
// Query vectors per KV head of a request that the few-rows kernel takes, which reads its keys once per 16 of them (us, few / tall: 64 vectors behind 4096 17 / 21, of 16
// requests behind 2000 49 / 49; 128 vectors 22 / 23 and 88 / 55).
constexpr int PAGED_FEW = 64;
// Shortest key ranges (few, us at 64 / 128 / 256: one row behind 100 8.2 / 6.7 / 6.7, behind 1024 10.2 / 9.2 / 10.3; tall, at 256 / 512 / 1024: a chunk of 316 rows beside
// 14 single tokens, 14/2 heads of 64, 22 / 24 / 34, 64 rows behind 4096 27 / 30 / 43)
constexpr int PAGED_KEYS_FEW = 128, PAGED_KEYS_TALL = 256;

// Rows of a request as the kernels read them: none where the lengths do not fit the buffers or the tables.  `descends` is set where cu does not ascend from 0 on: as
// long as it does, requests share no rows, and what they bring together fits max_rows, which the grids and the workspace are made for.
struct PagedReq { int first, n, start; };
__device__ __forceinline__ PagedReq paged_req(const PagedView& pv, int first, int end, int start, int max_new, bool& descends) {
  descends |= first < 0 || end < first;
  PagedReq q{first, (int)((unsigned)end - (unsigned)first), start};
  if (q.first < 0 || q.n < 0 || q.n > max_new || q.first > pv.max_rows - q.n || q.start < 0 || q.start > pv.limit - q.n) q.n = 0;
  return q;
}
__device__ __forceinline__ PagedReq paged_req(const PagedView& pv, const int* cu, const int* start, int max_new, int i, bool& descends) {
  return paged_req(pv, cu[i], cu[i + 1], start[i], max_new, descends);
}

// Where a launch's results go: rows of the cache's type, or (PLANES) the two bf16 planes that the projections read, in their layout
struct PagedOut { void* out; bf16_t* lo; long ld; int blocked; };

struct PagedWork {
  int shift;            // log2 of the blocks per KV head that the key ranges are chosen for
  int* count;           // [groups with several ranges][nkv]: ranges that have ended; 0 between launches
  float* part;          // [ranges of such groups][nkv]: QVT x HD sums, then QVT x (maximum, sum of weights)
};

// A block's share: rows row0 .. row0 + r - 1 of the request (its first row in the step is `first`), the first of them at position pos0; keys kb .. ke - 1;
// the range's number of n of its group; where partial results and the count lie (in slots of all KV heads)
struct PagedItem { int req, first, row0, r, pos0, kb, ke, split, n, slot, group; };

// A block's share of a step with shared prefixes, as its plan holds it (attention_shared.hpp): keys kb .. ke - 1 of the table of request `req`; step 1: the rows row0 .. row0 + r - 1, of which
// row j is at position pos0 + j and sees the keys up to there; step 0: the rows list[row0] .. list[row0 + r - 1], each (row, position), which see all keys up to pos0.
// unit: where row 0's partial results go, -1: to the output.
struct SharedItem { int req, row0, r, pos0, kb, ke, unit, step; };
// What the blocks of such a step share: the rows' list, and room for partial results: per unit the sums of all query heads, then their (maximum, sum of weights)
struct SharedParts {
  const int2* list;
  float* part;
  long unit_floats;
  __device__ __forceinline__ int2 row(const SharedItem& it, int j) const { return it.step ? make_int2(it.row0 + j, it.pos0 + j) : list[it.row0 + j]; }
  __device__ __forceinline__ float* sums(int unit, int head, int hd) const { return part + (size_t)unit * unit_floats + (size_t)head * hd; }
  __device__ __forceinline__ float* weights(int unit, int nh, int head, int hd) const { return part + (size_t)unit * unit_floats + (size_t)nh * hd + 2 * head; }
};

// The tall kernel's order of n items per KV head.  A chunk's later groups see more keys.  Up to PAGED_RESIDENT_TALL blocks are all resident from the start, two
// on a CU: the first round of the CUs goes from the longest down, the second from the shortest up, and a CU's two come to about the same.
// More blocks than that start as others end, longest first.
__device__ __forceinline__ int paged_turn(int y, int n, int nkv) {
  const int down = n * nkv <= PAGED_RESIDENT_TALL ? min(n, (PAGED_RESIDENT_TALL / 2 + nkv - 1) / nkv) : n;
  return y < down ? n - 1 - y : (y < n ? y - down : y);
}
struct PagedShare { int groups, splits; };
__device__ __forceinline__ int paged_groups(const PagedReq& q, int GQ, int lo, int hi, int rpb) {
  return q.n > 0 && q.n * GQ > lo && q.n * GQ <= hi ? (q.n + rpb - 1) / rpb : 0;
}
// Item y of the launch that takes requests with lo < rows x GQ <= hi in groups of rpb rows.  All ranges have kps keys: with T = sum of groups x
// keys over the requests, kps >= T / 2^shift, so there are at most 2^shift + groups items; those of groups with several ranges (keys > kps, hence ceil(keys / kps) < 2
// keys / kps) are fewer than 2^(shift + 1), and such groups fewer than 2^shift: what the workspace holds.  Called by whole blocks.  GROUP: y counts the
// groups with several ranges instead (split and range of the result mean nothing).
// The few-rows kernel has a group's last ranges, which may be short, behind all others (LAST_APART): where its blocks are somewhat more than the CUs, the short ones share.
template <int NT, int STEP, bool GROUP, bool TALL = false>
__device__ __forceinline__ bool paged_find(const PagedView& pv, const int* cu, const int* start, int max_new, int GQ, int lo, int hi, int rpb, int shift, int min_keys,
                                           int y, PagedItem& it) {
  auto keys_of = [&](unsigned long long total) {
    const unsigned long long per = (total + (1ull << shift) - 1) >> shift;
    return (int)min(max((unsigned long long)min_keys, (per + STEP - 1) / STEP * STEP), 1ull << 30);      // no request is longer
  };
  constexpr bool LAST_APART = !GROUP && !TALL;
  bool last = false;
  int i, kps, splits, before, slots, multi;
  PagedReq q;
  if (pv.n_req <= 64) {       // a request per lane, every wave for itself
    const int lane = threadIdx.x & 63;
    q = PagedReq{0, 0, 0};
    bool descends = false;
    if (lane < pv.n_req) q = paged_req(pv, cu, start, max_new, lane, descends);
    if (__any(descends)) return false;
    const int gr = paged_groups(q, GQ, lo, hi, rpb);
    kps = keys_of(wave_reduce((unsigned long long)gr * (unsigned)(q.start + q.n), [](unsigned long long a, unsigned long long b) { return a + b; }));
    const int sp = (int)((unsigned)(q.start + q.n + kps - 1) / (unsigned)kps);
    int items = GROUP ? (sp > 1 ? gr : 0) : LAST_APART ? gr * (sp - 1) : gr * sp;
    int incl = wave_scan(items);
    if (TALL) y = paged_turn(y, __builtin_amdgcn_readlane(incl, 63), pv.nkv);
    if (LAST_APART) {
      const int whole = __builtin_amdgcn_readlane(incl, 63);
      if (y >= whole) {
        y -= whole;
        last = true;
        items = gr;
        incl = wave_scan(items);
      }
    }
    const unsigned long long behind = __ballot(incl > y);
    if (!behind) return false;
    i = __builtin_ctzll(behind);
    const bool m = lane < i && sp > 1;
    slots = (int)wave_reduce((uint32_t)(m ? gr * sp : 0), [](uint32_t a, uint32_t b) { return a + b; });
    multi = (int)wave_reduce((uint32_t)(m ? gr : 0), [](uint32_t a, uint32_t b) { return a + b; });
    before = __builtin_amdgcn_readlane(incl - items, i);
    splits = __builtin_amdgcn_readlane(sp, i);
    q.first = __builtin_amdgcn_readlane(q.first, i);
    q.n = __builtin_amdgcn_readlane(q.n, i);
    q.start = __builtin_amdgcn_readlane(q.start, i);
  } else {
    __shared__ long long sums_s[NT / 64];
    __shared__ int found_s[8];
    const int tid = threadIdx.x, ipt = (pv.n_req + NT - 1) / NT, i0 = min(tid * ipt, pv.n_req), i1 = min(i0 + ipt, pv.n_req);
    long long mine = 0, total;
    bool descends = false;
    for (int j = i0; j < i1; ++j) {
      const PagedReq r = paged_req(pv, cu, start, max_new, j, descends);
      mine += (long long)paged_groups(r, GQ, lo, hi, rpb) * (r.start + r.n);
    }
    // rows are at most 2^24, keys 2^30: a sum of 2^55 and more says that some thread saw cu descend
    (void)block_scan<NT>(descends ? 1ll << 55 : mine, sums_s, total);
    if ((unsigned long long)total >> 55) return false;
    kps = keys_of((unsigned long long)total);
    // items in the low half, those of groups with several ranges in the upper one, and such groups
    long long n_items = 0, n_multi = 0;
    auto share = [&](int j) {
      const PagedReq r = paged_req(pv, cu, start, max_new, j, descends);
      return PagedShare{paged_groups(r, GQ, lo, hi, rpb), (int)((unsigned)(r.start + r.n + kps - 1) / (unsigned)kps)};
    };
    for (int j = i0; j < i1; ++j) {
      const PagedShare s = share(j);
      n_items += GROUP ? (s.splits > 1 ? s.groups : 0) : LAST_APART ? ((long long)s.groups << 32) + s.groups * (s.splits - 1) : (long long)s.groups * s.splits;
      if (s.splits > 1) n_multi += ((long long)s.groups << 32) | (unsigned)(s.groups * s.splits);
    }
    long long all, all_multi;
    long long at = block_scan<NT>(n_items, sums_s, all), at_multi = block_scan<NT>(n_multi, sums_s, all_multi);
    if (TALL) y = paged_turn(y, (int)all, pv.nkv);
    if (LAST_APART) {      // (the ranges in the low half, the last ones in the upper half)
      const int whole = (int)(all & 0xFFFFFFFF);
      last = y >= whole;
      y -= last ? whole : 0;
      all = last ? all >> 32 : whole;
      at = last ? at >> 32 : at & 0xFFFFFFFF;
      n_items = last ? n_items >> 32 : n_items & 0xFFFFFFFF;
    }
    if (y >= all) return false;
    if (at <= y && y < at + n_items) {
      for (int j = i0; j < i1; ++j) {
        const PagedShare s = share(j);
        const int n = GROUP ? (s.splits > 1 ? s.groups : 0) : LAST_APART ? s.groups * (last ? 1 : s.splits - 1) : s.groups * s.splits;
        if (y < at + n) {
          found_s[0] = j; found_s[1] = s.splits; found_s[2] = (int)at; found_s[3] = (int)(at_multi & 0xFFFFFFFF); found_s[4] = (int)(at_multi >> 32);
          break;
        }
        at += n;
        if (s.splits > 1) at_multi += ((long long)s.groups << 32) | (unsigned)(s.groups * s.splits);
      }
    }
    __syncthreads();
    i = __builtin_amdgcn_readfirstlane(found_s[0]);
    splits = found_s[1]; before = found_s[2]; slots = found_s[3]; multi = found_s[4];
    q = paged_req(pv, cu, start, max_new, i, descends);
  }
  // the same in every lane: in scalar registers from here on
  kps = __builtin_amdgcn_readfirstlane(kps);
  splits = __builtin_amdgcn_readfirstlane(splits);
  before = __builtin_amdgcn_readfirstlane(before);
  slots = __builtin_amdgcn_readfirstlane(slots);
  multi = __builtin_amdgcn_readfirstlane(multi);
  q = PagedReq{__builtin_amdgcn_readfirstlane(q.first), __builtin_amdgcn_readfirstlane(q.n), __builtin_amdgcn_readfirstlane(q.start)};
  const int per_group = LAST_APART ? (last ? 1 : splits - 1) : splits;
  const int rel = y - before, group = GROUP ? rel : (int)((unsigned)rel / (unsigned)per_group);
  it.req = i;
  it.first = q.first;
  it.row0 = group * rpb;
  it.r = min(rpb, q.n - it.row0);
  it.pos0 = q.start + it.row0;
  it.split = GROUP ? 0 : LAST_APART && last ? splits - 1 : rel - group * per_group;
  it.kb = it.split * kps;
  const int end = it.pos0 + it.r;                   // the group's last row sees the keys in front of this
  it.ke = min(end, it.kb + kps);
  it.n = (int)((unsigned)(end + kps - 1) / (unsigned)kps);      // of the request's ranges, those the group sees
  it.slot = slots + group * splits;
  it.group = multi + group;
  return it.kb < it.ke;
}

// Partial results pass from block to block, maybe from die to die, whose L2 caches do not see each other's lines.  They are written through
// those caches and read past them, 8 bytes at a time, by relaxed atomics of the device's scope; a fence of that scope would write a whole L2 back for each block that
// writes (31 single tokens behind up to 2111 keys: 204 us with such fences, 26 without) and empty it for each that joins (32 behind 2048, 14/2 heads of 64: 16.7, 13.5).
__device__ __forceinline__ void put_through(float* p, float a, float b) {
  __hip_atomic_store((unsigned long long*)p, ((unsigned long long)__float_as_uint(b) << 32) | __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_past(const float* p) {
  const unsigned long long v = __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
__device__ __forceinline__ void put_through4(float* p, const f32x4& v) { put_through(p, v.x, v.y); put_through(p + 2, v.z, v.w); }

// 4 dims of a vector summed over ranges: o = sum of weights x values and l = sum of weights, both relative to the maximum m (powers of two)
struct PagedSum {
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(float m2, float l2, const f32x4& o2) {
    const float mn = fmaxf(m, m2), mu = mn == -INFINITY ? 0.f : mn, f = __builtin_amdgcn_exp2f(m - mu), f2 = __builtin_amdgcn_exp2f(m2 - mu);
    l = l * f + l2 * f2;
    o = f * o + f2 * o2;
    m = mn;
  }
  // ranges s0, s0 + by, ... below n, of partial results `step` floats apart (PAST: put through by blocks of the same launch)
  template <bool PAST>
  __device__ __forceinline__ void add_ranges(const float* ml, const float* po, size_t step, int s0, int n, int by) {
    constexpr int U = 8;                  // of them in flight
    for (; s0 < n; s0 += U * by) {
      float2 w[U];
      f32x4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t at = (size_t)min(s0 + u * by, n - 1) * step;
        if (PAST) {
          const float2 a = get_past(po + at), b = get_past(po + at + 2);
          w[u] = get_past(ml + at);
          x[u] = f32x4{a.x, a.y, b.x, b.y};
        } else {
          w[u] = *(const float2*)(ml + at);
          x[u] = *(const f32x4*)(po + at);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (s0 + u * by < n) add(w[u].x, w[u].y, x[u]);
    }
  }
  __device__ __forceinline__ f32x4 result() const {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    return f32x4{o.x * inv, o.y * inv, o.z * inv, o.w * inv};
  }
};

// The end of a block whose group has several ranges: `write` has stored the block's partial results in its slot; the last of the group's blocks joins
// all of them.  o: QVT x HD sums relative to the maximum m (powers of two), l: sum of weights; out = sum 2^(m - M) o / sum 2^(m - M) l.
// A wave waits for its writes before the block counts.
template <int HD, int QVT, int NT, typename STORE>
__device__ __forceinline__ void paged_join(const PagedWork& w, const PagedItem& it, int nkv, int g, int QV, f32x4* sums /* LDS, 2 NT of them */, STORE store) {
  __shared__ int last_s;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  const int tid = threadIdx.x;
  if (tid == 0) {
    int* c = w.count + (size_t)it.group * nkv + g;
    last_s = __hip_atomic_fetch_add(c, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == it.n - 1;
    if (last_s) __hip_atomic_store(c, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last_s) return;
  constexpr size_t SLOT = (size_t)QVT * (HD + 2);
  const float* part = w.part + ((size_t)it.slot * nkv + g) * SLOT;
  const size_t step = (size_t)nkv * SLOT;
  // 4 dims of a vector a thread; where the vectors are few, several threads share the ranges of one and meet in LDS, in their order
  constexpr int T4 = HD / 4;
  const int cells = QV * T4;
  int share = 1;
  while (2 * share * cells <= NT && 2 * share <= it.n) share *= 2;
  for (int e0 = 0; e0 < cells; e0 += NT) {
    const int e = e0 + tid, turn = share > 1 ? e / cells : 0, cell = share > 1 ? e - turn * cells : e;
    const bool on = turn < share && cell < cells;
    const int v = on ? cell / T4 : 0, d = on ? (cell % T4) * 4 : 0;
    PagedSum sum;
    sum.add_ranges<true>(part + (size_t)QVT * HD + 2 * v, part + (size_t)v * HD + d, step, on ? turn : it.n, it.n, share);
    if (share > 1) {
      sums[tid] = sum.o;
      sums[NT + tid] = f32x4{sum.m, sum.l, 0.f, 0.f};
      __syncthreads();
      if (turn == 0 && on)
        for (int k = 1; k < share; ++k) sum.add(sums[NT + k * cells + cell].x, sums[NT + k * cells + cell].y, sums[k * cells + cell]);
    }
    if (on && turn == 0) store(v, d, sum.result());
  }
}

// Four values of one head from dim d on, rounded once
template <typename CT, bool PLANES>
__device__ __forceinline__ void paged_store4(const PagedOut& o, int row, int col, const f32x4& v) {
  if (PLANES) {
    const size_t at = packed_at(o.blocked, row, col, (int)o.ld);
    const uint2 h = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    *(uint2*)((bf16_t*)o.out + at) = h;
    *(uint2*)(o.lo + at) = make_uint2(pack_bf16x2(v.x - __uint_as_float(h.x << 16), v.y - __uint_as_float(h.x & 0xFFFF0000u)),
                                      pack_bf16x2(v.z - __uint_as_float(h.y << 16), v.w - __uint_as_float(h.y & 0xFFFF0000u)));
  } else if (sizeof(CT) == 4) {
    *(f32x4*)((float*)o.out + (size_t)row * o.ld + col) = v;
  } else {
    *(uint2*)((bf16_t*)o.out + (size_t)row * o.ld + col) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
  }
}

// A pair of probabilities in two bf16 parts
__device__ __forceinline__ void paged_split2(float a, float b, uint32_t& h, uint32_t& l) {
  h = pack_bf16x2(a, b);
  l = pack_bf16x2(a - __uint_as_float(h << 16), b - __uint_as_float(h & 0xFFFF0000u));
}

// Groups of 16 keys that a wave has under way, and weighs with one maximum: 8 KiB of bf16, and twice that where a wave works alone, with fewer of them on a CU.
template <typename CT, bool SHARED> __host__ __device__ constexpr int paged_few_groups() { return sizeof(CT) == 4 ? 1 : sizeof(CT) == 1 || SHARED ? 2 : 1; }

// Requests with few query vectors.  16 vectors of one KV head are the 16 columns of the matrix tiles, so a block reads each key and value once; its 4
// waves take groups of 16 keys in turn, which never leave a page, the next group's loads in flight.  Per group, in one wave (lane: sl = lane % 16, kq = lane / 16):
//   scores   S^T[key, q] = sum_d K[key, d] Q[q, d], 16x16x32: K rows as they lie in the cache, the queries as two bf16 parts (16 bits);
//   output   O[q, d] += sum_key P[q, key] V[key, d], 16x16x16: a lane's operand is 4 consecutive keys of one row or column, so nothing moves between
//            lanes; a probability goes in as PAGED_PARTS bf16 parts.
// fp32 caches: 16x16x4 for both, the queries and probabilities as they are, any number of rows (a chunk's groups of 16 vectors find the keys in the L2).
// Values are loaded past the L2, keys through it: a key's 256 bytes take four loads, which share cache lines (us, both through the caches / values past
// them / both: 3 rows of 8 requests behind 16384 102 / 84 / 91, 31 ragged rows in pages of 16 tokens 23 / 25 / 30, out of cold memory 29 / 28 / 30, one row of 64
// behind 1024 out of cold memory 54 / 49 / 48).
// Bound by the memory: 8 KiB per wave and group against PAGED_PARTS x HD / 16 + 2 x HD / 32 products.
// SHARED: `it` is a SharedItem, a wave's alone (`slot`: its number in the block, tid its lane): no barriers, and the wave's own result is the item's, to go where it says.
template <typename CT, int HD, bool PLANES, bool SHARED, typename ITEM>
__device__ __forceinline__ void paged_few_item(const ITEM& it, int g, const int tid, int slot, const float* __restrict__ qkv, long ld, const typename PagedWide<CT>::type* __restrict__ q_gain,
                                               const float2* __restrict__ rope_tab, float eps, const PagedOut& po, const PagedView& pv, const PagedWork& wk, const SharedParts& sp) {
  typedef typename PagedWide<CT>::type GT;
  constexpr bool BF = sizeof(GT) == 2, Q8 = sizeof(CT) == 1;
  constexpr int PARTS = PAGED_PARTS<PLANES>;
  constexpr int QVT = 16, NW = SHARED ? 1 : PAGED_WAVES, NT = 64 * NW, DPL = HD / 16, half = HD / 2, HL = HD / 32;
  constexpr int QI = 16 * QVT / NT;                          // query vectors that 16 lanes make ready
  constexpr int KS = HD * (int)sizeof(CT) / 64;              // 16-byte pieces of a key a lane carries
  constexpr int G = paged_few_groups<CT, SHARED>();          // groups of 16 keys that a wave loads and weighs together
  constexpr int QLD = BF ? HD + ATT_QPAD : HD + 4;           // a query row in LDS
  constexpr int KW = BF ? HD / 32 : HD / 16;                 // pieces of a key in the products: KS, or 8-bit ones widened
  constexpr int VW = DPL * sizeof(GT) / 4;                   // 32-bit words of a value in the products: its DPL dims that a lane carries
  typedef unsigned int vraw_t __attribute__((ext_vector_type(Q8 ? VW / 2 : VW)));
  typedef unsigned int vwide_t __attribute__((ext_vector_type(VW)));
  typedef float fvec_t __attribute__((ext_vector_type(HL)));
  typedef unsigned short hvec_t __attribute__((ext_vector_type(HL)));
  const int GQ = pv.gq;
  const int lane = tid & 63, wave = SHARED ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6), sl = lane & 15, kq = lane >> 4;
  const int QV = it.r * GQ, ke = it.ke;
  __shared__ float wm[NW][QVT], wl[NW][QVT];
  __shared__ int poison_s;
  extern __shared__ float4 paged_dyn_smem[];
  float* wacc = (float*)paged_dyn_smem;                       // [NW][QV][HD], in the place of the queries' two parts when these are done with
  GT (*qhi_s)[QLD] = (GT (*)[QLD])paged_dyn_smem + slot * (BF ? 2 : 1) * QVT, (*qlo_s)[QLD] = qhi_s + QVT;      // (fp32: one part)
  // pages of this wave's next 64 groups, one a lane
  const int* trow = pv.table + (size_t)it.req * pv.max_pages;
  auto load_pages = [&](int base) { return base + 16 * NW * lane < ke ? trow[(base + 16 * NW * lane) >> pv.page_shift] : 0; };
  const int first = it.kb + 16 * wave;
  int pages = load_pages(first);
  // query vectors tid / 16 + 4 i, 2 HL values a lane
  const int l16 = tid & 15;
  fvec_t xa[QI], xb[QI];
  float2 cs[QI][HL];
  GT g0[HL], g1[HL];
#pragma unroll
  for (int e = 0; e < HL; ++e) {
    g0[e] = q_gain ? q_gain[HL * l16 + e] : GT(0);
    g1[e] = q_gain ? q_gain[half + HL * l16 + e] : GT(0);
  }
#pragma unroll
  for (int i = 0; i < QI; ++i) {
    // what it needs is asked for in front of the keys, whose arrival it is made ready beside
    if (i > 0 && i * NT / 16 >= QV) break;
    const int qv = (tid >> 4) + i * (NT / 16), qr = pv.row_of(qv < QV ? qv : 0), qrow = it.row0 + qr, qhead = g * GQ + (qv < QV ? qv - qr * GQ : 0);
    int row, pos;
    if constexpr (SHARED) { const int2 rp = sp.row(it, qr); row = rp.x; pos = rp.y; }
    else { row = it.first + qrow; pos = it.pos0 + qr; }
    const float* src = qkv + (size_t)row * ld + (size_t)qhead * HD + HL * l16;
    xa[i] = *(const fvec_t*)src; xb[i] = *(const fvec_t*)(src + half);
    const float2* rp = rope_tab + (size_t)pos * half + HL * l16;
#pragma unroll
    for (int e = 0; e < HL; ++e) cs[i][e] = rope_tab ? rp[e] : make_float2(1.f, 0.f);
  }
  int poison = INT_MAX;      // SHARED: the least key of this lane's whose value is not finite, among those that some row does not see
  if (!SHARED && tid == 0) poison_s = INT_MAX;
  u32x4 kr[G][KS];
  vraw_t vr[G][4];
  bool ok[G];
  uint32_t ksr[G], vsr[G];                                    // 8 bits: the scale of the lane's key, those of its four values
  auto load_kv = [&](int base, int page, int u) {
    ok[u] = page >= 0 && page < pv.n_pages;
    const size_t row = ((size_t)g << pv.page_shift) + (base & ((1 << pv.page_shift) - 1));
    const size_t at = (size_t)(ok[u] ? page : 0) * pv.page_stride + row * HD;
    const CT* kp = (const CT*)pv.k + at;
    const CT* vp = (const CT*)pv.v + at;
#pragma unroll
    for (int t = 0; t < KS; ++t) kr[u][t] = *(const u32x4*)(kp + sl * HD + (HD / KS) * t + (16 / (int)sizeof(CT)) * kq);
#pragma unroll
    for (int m = 0; m < 4; ++m) vr[u][m] = __builtin_nontemporal_load((const vraw_t*)(vp + (4 * kq + m) * HD + DPL * sl));
    if constexpr (Q8) {
      const size_t sc = (size_t)(ok[u] ? page : 0) * pv.scale_stride + row;
      ksr[u] = pv.ks[sc + sl];
      vsr[u] = *(const uint32_t*)(pv.vs + sc + 4 * kq);
    }
  };
  // groups j .. j + G - 1 of this wave's (load_pages(base) has been called for 64 of them)
  auto load_groups = [&](int base, int j) {
#pragma unroll
    for (int u = 0; u < G; ++u) {
      const bool in = u == 0 || base + 16 * NW * u < ke;      // (in place of one behind the last key the first one again, which counts for nothing)
      load_kv(in ? base + 16 * NW * u : base, __builtin_amdgcn_readlane(pages, (in ? j + u : j) & 63), u);
      ok[u] &= in;
    }
  };
  if (first < ke) load_groups(first, 0);
#pragma unroll
  for (int i = 0; i < QI; ++i) {
    if (i > 0 && i * NT / 16 >= QV) break;      // (columns of the products behind the last vector hold whatever lies there)
    const int qv = (tid >> 4) + i * (NT / 16);
    float x0[HL], x1[HL], ss = 0.f;
#pragma unroll
    for (int e = 0; e < HL; ++e) { x0[e] = xa[i][e]; x1[e] = xb[i][e]; ss += __builtin_fmaf(x0[e], x0[e], x1[e] * x1[e]); }      // (written out, as the rotation below)
    if (q_gain) {
      const float rs = rsqrtf(row16_sum(ss) / (float)HD + eps);
#pragma unroll
      for (int e = 0; e < HL; ++e) { x0[e] *= rs * Elem<GT>::to_f32(g0[e]); x1[e] *= rs * Elem<GT>::to_f32(g1[e]); }
    }
    if (rope_tab) {
#pragma unroll
      for (int e = 0; e < HL; ++e) {      // (which product is the rounded one is written out: the compiler's own choice differs from one instantiation to the next)
        const float a = x0[e], b = x1[e];
        x0[e] = __builtin_fmaf(a, cs[i][e].x, -(b * cs[i][e].y));
        x1[e] = __builtin_fmaf(a, cs[i][e].y, b * cs[i][e].x);
      }
    }
    const float scale = rsqrtf((float)HD) * 1.4426950408889634f;
    if constexpr (BF) {
      hvec_t h0, h1, l0, l1;
#pragma unroll
      for (int e = 0; e < HL; ++e) {
        bf16_t h, l;
        split_bf16(qv < QV ? x0[e] * scale : 0.f, h, l); h0[e] = h; l0[e] = l;
        split_bf16(qv < QV ? x1[e] * scale : 0.f, h, l); h1[e] = h; l1[e] = l;
      }
      *(hvec_t*)&qhi_s[qv][HL * l16] = h0; *(hvec_t*)&qhi_s[qv][half + HL * l16] = h1;
      *(hvec_t*)&qlo_s[qv][HL * l16] = l0; *(hvec_t*)&qlo_s[qv][half + HL * l16] = l1;
    } else {
#pragma unroll
      for (int e = 0; e < HL; ++e) { qhi_s[qv][HL * l16 + e] = qv < QV ? x0[e] * scale : 0.f; qhi_s[qv][half + HL * l16 + e] = qv < QV ? x1[e] * scale : 0.f; }
    }
  }
  if constexpr (SHARED) {      // a wave's LDS accesses are in order: only the compiler has to keep them so
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  } else {
    __syncthreads();
  }
  int my_pos = it.pos0 + pv.row_of(sl);
  if constexpr (SHARED) my_pos = it.step ? my_pos : it.pos0;
  float m_run = -INFINITY, l_run = 0.f;
  f32x4 acc[DPL];
#pragma unroll
  for (int e = 0; e < DPL; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto rescale = [&](float f) {                               // the sums this lane holds are those of queries 4 kq + j
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float fq = __shfl(f, 4 * kq + q, 64);
#pragma unroll
      for (int e = 0; e < DPL; ++e) acc[e][q] *= fq;
    }
  };
  auto not_finite = [&](const vwide_t& v) {
    bool bad = false;
#pragma unroll
    for (int u = 0; u < VW; ++u) bad |= (BF && (v[u] & 0x7F80u) == 0x7F80u) || (v[u] & 0x7F800000u) == 0x7F800000u;
    return bad;
  };
  if constexpr (G == 1) {
    for (int base = first, j = 0; base < ke; base += 16 * NW, ++j) {
      u32x4 ka[KS];
      vwide_t va[4];
      const bool here = ok[0];
#pragma unroll
      for (int t = 0; t < KS; ++t) ka[t] = kr[0][t];
#pragma unroll
      for (int m = 0; m < 4; ++m) va[m] = __builtin_bit_cast(vwide_t, vr[0][m]);
      const int next = base + 16 * NW;
      if (next < ke) {
        if ((j & 63) == 63) pages = load_pages(next);
        load_groups(next, j + 1);
      }
      if (!here) continue;                                      // a page outside the pool
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        if constexpr (!BF) {
          const f32x4 k4 = __builtin_bit_cast(f32x4, ka[t]), q4 = *(const f32x4*)&qhi_s[sl][16 * t + 4 * kq];
#pragma unroll
          for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k4[e], q4[e], s, 0, 0, 0);
          continue;
        } else {
          const bf16x8_t ql = __builtin_bit_cast(bf16x8_t, *(const u32x4*)&qlo_s[sl][32 * t + 8 * kq]), qh = __builtin_bit_cast(bf16x8_t, *(const u32x4*)&qhi_s[sl][32 * t + 8 * kq]);
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ka[t]), ql, s, 0, 0, 0);
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ka[t]), qh, s, 0, 0, 0);
        }
      }
      float sc[4] = {s.x, s.y, s.z, s.w};
      if (base + 16 > it.pos0 + 1) {
        // Keys that some row does not see: their scores are out; values behind the last key are whatever lies there, and values of the item's own
        // positions may be infinite or NaN, which a probability of 0 would not silence: both go in as 0, and the rows that see such a one become NaN
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const int key = base + 4 * kq + m;
          if (key > my_pos || key >= ke) sc[m] = -INFINITY;
          if (key > it.pos0) {
            const bool bad = not_finite(va[m]);
            if (bad && key < ke) {
              if constexpr (SHARED) poison = min(poison, key);
              else atomicMin(&poison_s, key);
            }
            if (bad || key >= ke) va[m] = vwide_t(0u);
          }
        }
      }
      float mx = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3]));
      mx = column_max(mx);
      const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float f = __builtin_amdgcn_exp2f(m_run - m_use);
      float p[4];
      float psum = 0.f;
#pragma unroll
      for (int m = 0; m < 4; ++m) { p[m] = __builtin_amdgcn_exp2f(sc[m] - m_use); psum += p[m]; }
      l_run = l_run * f + psum;
      if (__any(m_new > m_run)) rescale(f);
      m_run = m_new;
      if constexpr (!BF) {
#pragma unroll
        for (int e = 0; e < DPL; ++e)
#pragma unroll
          for (int m = 0; m < 4; ++m) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[m], __uint_as_float(va[m][e]), acc[e], 0, 0, 0);
      } else {
        uint2 pp[PARTS];
        if constexpr (PARTS == 3) {
          paged_split3(p[0], p[1], pp[0].x, pp[1].x, pp[2].x);
          paged_split3(p[2], p[3], pp[0].y, pp[1].y, pp[2].y);
        } else {
          paged_split2(p[0], p[1], pp[0].x, pp[1].x);
          paged_split2(p[2], p[3], pp[0].y, pp[1].y);
        }
#pragma unroll
        for (int e = 0; e < DPL; ++e) {
          const unsigned int sel = (e & 1) ? 0x07060302u : 0x05040100u;
          const uint2 v4 = make_uint2(__builtin_amdgcn_perm(va[1][e >> 1], va[0][e >> 1], sel), __builtin_amdgcn_perm(va[3][e >> 1], va[2][e >> 1], sel));
#pragma unroll
          for (int z = PARTS - 1; z >= 0; --z)
            acc[e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(bf16x4s_t, pp[z]), __builtin_bit_cast(bf16x4s_t, v4), acc[e], 0, 0, 0);
        }
      }
    }
  } else if constexpr (BF) {
    // G groups at once: the queries stay in registers, the groups' scores are chains that do not wait for each other, one maximum serves all, and the values enter by pairs of groups
    // (16x16x32: a lane's eight keys are four of either).  8-bit pieces are 16 consecutive dims of a key a lane, and the products' eight go by that.
    static_assert(PARTS == 2 && G % 2 == 0, "two parts of a probability, pairs of groups");
    bf16x8_t qh[KW], ql[KW];
#pragma unroll
    for (int t = 0; t < KW; ++t) {
      const int d0 = Q8 ? 64 * (t >> 1) + 16 * kq + 8 * (t & 1) : 32 * t + 8 * kq;
      qh[t] = __builtin_bit_cast(bf16x8_t, *(const u32x4*)&qhi_s[sl][d0]);
      ql[t] = __builtin_bit_cast(bf16x8_t, *(const u32x4*)&qlo_s[sl][d0]);
    }
    for (int from = first, j = 0; from < ke; from += 16 * NW * G, j += G) {
      u32x4 kc[G][KS];
      vraw_t vc[G][4];
      bool here[G], all = true, some = false;
      uint32_t ksc[G], vsc[G];
#pragma unroll
      for (int u = 0; u < G; ++u) {
        here[u] = ok[u];
        all &= ok[u];
        some |= ok[u];
#pragma unroll
        for (int t = 0; t < KS; ++t) kc[u][t] = kr[u][t];
#pragma unroll
        for (int m = 0; m < 4; ++m) vc[u][m] = vr[u][m];
        if constexpr (Q8) { ksc[u] = ksr[u]; vsc[u] = vsr[u]; }
      }
      const int next = from + 16 * NW * G;
      if (next < ke) {
        if (((j + G) & 63) == 0) pages = load_pages(next);
        load_groups(next, j + G);
      }
      if (!some) continue;                                      // pages outside the pool
      f32x4 s[G];
#pragma unroll
      for (int u = 0; u < G; ++u) s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        constexpr int STEPS = Q8 ? 2 : 1;
        bf16x8_t k8[G][STEPS];
#pragma unroll
        for (int u = 0; u < G; ++u) {
          if constexpr (Q8) {
            const float sk = e8m0_scale(ksc[u]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
              k8[u][h] = __builtin_bit_cast(bf16x8_t, u32x4{e4m3_pair<false>(kc[u][t][2 * h], sk), e4m3_pair<true>(kc[u][t][2 * h], sk), e4m3_pair<false>(kc[u][t][2 * h + 1], sk),
                                                            e4m3_pair<true>(kc[u][t][2 * h + 1], sk)});
          } else {
            k8[u][0] = __builtin_bit_cast(bf16x8_t, kc[u][t]);
          }
        }
#pragma unroll
        for (int h = 0; h < STEPS; ++h) {
#pragma unroll
          for (int u = 0; u < G; ++u) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8[u][h], ql[STEPS * t + h], s[u], 0, 0, 0);
#pragma unroll
          for (int u = 0; u < G; ++u) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8[u][h], qh[STEPS * t + h], s[u], 0, 0, 0);
        }
      }
      const bool edge = next > it.pos0 + 1;                     // keys that some row does not see
      if (edge || !all) {
#pragma unroll
        for (int u = 0; u < G; ++u)
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const int key = from + 16 * NW * u + 4 * kq + m;
            if (!here[u] || key > my_pos || key >= ke) s[u][m] = -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < G; ++u) mx = fmaxf(mx, fmaxf(fmaxf(s[u][0], s[u][1]), fmaxf(s[u][2], s[u][3])));
      mx = column_max(mx);
      const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float f = __builtin_amdgcn_exp2f(m_run - m_use);
      float psum = 0.f;
      uint32_t ph[G][2], pl[G][2];
#pragma unroll
      for (int u = 0; u < G; ++u) {
        float p[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) { p[m] = __builtin_amdgcn_exp2f(s[u][m] - m_use); psum += p[m]; }
        paged_split2(p[0], p[1], ph[u][0], pl[u][0]);
        paged_split2(p[2], p[3], ph[u][1], pl[u][1]);
      }
      l_run = l_run * f + psum;
      if (__any(m_new > m_run)) rescale(f);
      m_run = m_new;
#pragma unroll
      for (int u0 = 0; u0 < G; u0 += 2) {
        vwide_t va[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            if constexpr (Q8) {
              const float sv = e8m0_scale((vsc[u0 + i] >> (8 * m)) & 0xFFu);
#pragma unroll
              for (int e = 0; e < VW / 2; ++e) { va[i][m][2 * e] = e4m3_pair<false>(vc[u0 + i][m][e], sv); va[i][m][2 * e + 1] = e4m3_pair<true>(vc[u0 + i][m][e], sv); }
            } else {
              va[i][m] = __builtin_bit_cast(vwide_t, vc[u0 + i][m]);
            }
          }
        if (edge || !all) {                                     // (what is silenced here, and why: as above)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              const int key = from + 16 * NW * (u0 + i) + 4 * kq + m;
              const bool bad = key > it.pos0 && not_finite(va[i][m]);
              if (bad && here[u0 + i] && key < ke) {
                if constexpr (SHARED) poison = min(poison, key);
                else atomicMin(&poison_s, key);
              }
              if (bad || !here[u0 + i] || key >= ke) va[i][m] = vwide_t(0u);
            }
        }
#pragma unroll
        for (int e = 0; e < DPL; ++e) {
          const unsigned int sel = (e & 1) ? 0x07060302u : 0x05040100u;
          const bf16x8_t v8 = __builtin_bit_cast(bf16x8_t, u32x4{__builtin_amdgcn_perm(va[0][1][e >> 1], va[0][0][e >> 1], sel), __builtin_amdgcn_perm(va[0][3][e >> 1], va[0][2][e >> 1], sel),
                                                                 __builtin_amdgcn_perm(va[1][1][e >> 1], va[1][0][e >> 1], sel), __builtin_amdgcn_perm(va[1][3][e >> 1], va[1][2][e >> 1], sel)});
          acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, u32x4{pl[u0][0], pl[u0][1], pl[u0 + 1][0], pl[u0 + 1][1]}), v8, acc[e], 0, 0, 0);
          acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, u32x4{ph[u0][0], ph[u0][1], ph[u0 + 1][0], ph[u0 + 1][1]}), v8, acc[e], 0, 0, 0);
        }
      }
    }
  }
  l_run = column_sum(l_run);
  if constexpr (SHARED) {
    poison = wave_reduce((uint32_t)poison, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
    if (it.pos0 + pv.row_of(sl) >= poison) l_run = __uint_as_float(0x7FC00000u);
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int v = 4 * kq + q, r = pv.row_of(v), head = g * GQ + v - r * GQ;
      const float inv_q = __shfl(inv, v, 64);
      if (v >= QV) continue;
      if (it.unit < 0) {
        const int row = sp.row(it, r).x;
#pragma unroll
        for (int e = 0; e < DPL; e += 4) paged_store4<GT, PLANES>(po, row, head * HD + DPL * sl + e, f32x4{acc[e][q] * inv_q, acc[e + 1][q] * inv_q, acc[e + 2][q] * inv_q, acc[e + 3][q] * inv_q});
      } else {
        float* sums = sp.sums(it.unit + r, head, HD) + DPL * sl;
#pragma unroll
        for (int e = 0; e < DPL; e += 4) *(f32x4*)(sums + e) = f32x4{acc[e][q], acc[e + 1][q], acc[e + 2][q], acc[e + 3][q]};
      }
    }
    if (it.unit >= 0 && kq == 0 && sl < QV) {
      const int r = pv.row_of(sl);
      *(float2*)sp.weights(it.unit + r, pv.nh, g * GQ + sl - r * GQ, HD) = make_float2(m_run, l_run);
    }
    return;
  } else {
    // the waves' results of a vector, 4 consecutive dims a thread
    __syncthreads();
    if (kq == 0 && sl < QV) { wm[wave][sl] = m_run; wl[wave][sl] = l_run; }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (4 * kq + q < QV) {
        float* dst = wacc + ((size_t)wave * QV + 4 * kq + q) * HD + DPL * sl;
#pragma unroll
        for (int e = 0; e < DPL; ++e) dst[e] = acc[e][q];
      }
    }
    __syncthreads();
    constexpr size_t SLOT = (size_t)QVT * (HD + 2);
    float* part = wk.part + ((size_t)(it.slot + it.split) * pv.nkv + g) * SLOT;
    auto store = [&](int v, int d, const f32x4& x) {
      const int r = pv.row_of(v);
      paged_store4<GT, PLANES>(po, it.first + it.row0 + r, (g * GQ + v - r * GQ) * HD + d, x);
    };
    for (int e = tid; e < QV * (HD / 4); e += NT) {
      const int v = e / (HD / 4), d = (e % (HD / 4)) * 4;
      float mm = wm[0][v];
#pragma unroll
      for (int w = 1; w < NW; ++w) mm = fmaxf(mm, wm[w][v]);
      const float mu = mm == -INFINITY ? 0.f : mm;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      float l = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float fw = __builtin_amdgcn_exp2f(wm[w][v] - mu);
        o += fw * *(const f32x4*)(wacc + ((size_t)w * QV + v) * HD + d);
        l += fw * wl[w][v];
      }
      if (it.pos0 + pv.row_of(v) >= poison_s) l = __uint_as_float(0x7FC00000u);
      if (it.n == 1) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        store(v, d, f32x4{o.x * inv, o.y * inv, o.z * inv, o.w * inv});
      } else {
        put_through4(part + (size_t)v * HD + d, o);
        if (d == 0) put_through(part + (size_t)QVT * HD + 2 * v, mm, l);
      }
    }
    if (it.n > 1) paged_join<HD, QVT, NT>(wk, it, pv.nkv, g, QV, (f32x4*)paged_dyn_smem, store);
  }
}

template <typename CT, int HD, bool PLANES>
__device__ __forceinline__ void paged_attention_few(int y, const int* __restrict__ cu, const int* __restrict__ start, const float* __restrict__ qkv, long ld,
                                                    const typename PagedWide<CT>::type* __restrict__ q_gain, const float2* __restrict__ rope_tab, float eps, int max_new, int hi, const PagedOut& po,
                                                    const PagedView& pv, const PagedWork& wk) {
  constexpr int NW = PAGED_WAVES, NT = 64 * NW;
  PagedItem it;
  if (!paged_find<NT, 16 * NW, false>(pv, cu, start, max_new, pv.gq, 0, hi, pv.rpb_few, wk.shift, PAGED_KEYS_FEW, y, it)) return;
  paged_few_item<CT, HD, PLANES, false>(it, blockIdx.x, threadIdx.x, 0, qkv, ld, q_gain, rope_tab, eps, po, pv, wk, SharedParts{});
}

// Requests with many query vectors (chunks of a prompt).  A block takes 128 vectors of one KV head - 128 / GQ rows x the GQ query heads that share it, 32 per
// wave - and walks its range of keys in tiles of 64 through LDS.  Per tile and wave, with 32x32x16 products:
//   scores   S^T[key, q]: K rows from LDS, the queries in registers as two bf16 parts; a lane ends up with 16 keys of one vector per 32 keys;
//   output   O^T[d, q] += sum_key V^T[d, key] P^T[key, q]: a lane's own probabilities are the operand as they stand, V^T comes from LDS; a
//            probability goes in as PAGED_PARTS bf16 parts.
// K goes from the pages straight into LDS, a wave 16 keys of a tile (one page), rows' 16-byte chunks permuted by the key number; V through registers, transposed
// on the way (4 keys x HD / 16 dims per thread; 8-byte pieces permuted by the dim).  Two buffers of each: the next tile's loads fly during
// a tile, and a tile's page numbers are fetched a tile earlier still, one per 4 keys and lane.
// The products run over whole tiles, with probability 0 for keys that a row does not see.  Values behind the block's last key go into LDS as 0.  Values of its
// own positions may be infinite or NaN, which 0 does not silence: the block looks at them first; if one is not finite, it and its like behind
// it go into LDS as 0 and the rows that see it become NaN.
template <typename CT, int HD, bool PLANES, bool SHARED, typename ITEM>
__device__ __forceinline__ void paged_tall_item(const ITEM& it, int g, const int tid, const float* __restrict__ qkv, long ld, const bf16_t* __restrict__ q_gain,
                                                const float2* __restrict__ rope_tab, float eps, const PagedOut& po, const PagedView& pv, const PagedWork& wk, const SharedParts& sp) {
  constexpr int PARTS = PAGED_PARTS<PLANES>;
  constexpr int QVT = 128, NT = 256, KT = 64;
  constexpr int T = HD / 16;           // steps over d for the scores
  constexpr int DT = HD / 32;          // 32-dim tiles of the output
  constexpr int DV = HD / 16;          // dims of V a thread carries
  constexpr int CH = HD / 8;           // 16-byte chunks of a K row
  constexpr bool Q8 = sizeof(CT) == 1;
  constexpr int KI = KT * CH / 256 / (Q8 ? 2 : 1);      // K pieces (16 bytes per lane) per wave and tile
  constexpr int TILE = KT * HD;
  constexpr int VR = Q8 ? DV / 4 : DV / 2;              // words of a value as they come from the pool
  typedef unsigned int vraw_t __attribute__((ext_vector_type(VR)));
  typedef unsigned int vwide_t __attribute__((ext_vector_type(DV / 2)));
  extern __shared__ float4 paged_dyn_smem[];
  __shared__ int poison_s;
  const int GQ = pv.gq;
  const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), hi = lane >> 5;
  // LDS by byte address: K, K, V^T, V^T from a multiple of 1 KiB on, so that a permuted piece's address is the row's with bits exclusive-or'ed in
  typedef __attribute__((address_space(3))) char lds_char;
  typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
  typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
  const uint32_t ring = ((uint32_t)(uintptr_t)(lds_char*)(char*)paged_dyn_smem + 1023u) & ~1023u;
  const int QV = it.r * GQ, qv = 32 * w + (lane & 31), kb = it.kb, ke = it.ke;
  const bool valid = qv < QV;
  const int qr = pv.row_of(valid ? qv : 0), row = it.row0 + qr, head = g * GQ + (valid ? qv - qr * GQ : 0);
  int my_pos = it.pos0 + (row - it.row0), qkv_row, rope_pos;
  if constexpr (SHARED) {
    const int2 rp = sp.row(it, qr);
    qkv_row = rp.x;
    rope_pos = rp.y;
    my_pos = it.step ? my_pos : it.pos0;
  } else {
    qkv_row = it.first + row;
    rope_pos = my_pos;
  }
  const int* trow = pv.table + (size_t)it.req * pv.max_pages;
  const int in_page = (1 << pv.page_shift) - 1;

  // the page of this lane's 4 keys of a tile (the last key's where they lie behind it)
  auto load_pages = [&](int base) { return trow[min(base + 4 * (lane & 15), ke - 1) >> pv.page_shift]; };
  auto outside = [&](int page) { return page < 0 || page >= pv.n_pages; };
  // K: piece i of the wave's 16 keys holds 64 / CH of them, a chunk of one per lane, permuted by the key number
  u32x4 kraw[Q8 ? KI : 1];
  uint32_t kscale = 0, vscale = 0;      // 8 bits: the scales of keys 4 (lane % 16) .. + 3 of the tile
  auto load_k = [&](int ln, int base, int page, int buf, int i) {
    if constexpr (Q8) {      // codes: into registers, 16 of one key a lane; store_k widens them into LDS
      const int pg = __builtin_amdgcn_readlane(page, 4 * w), key = (i * 64 + ln) / (HD / 16);
      const size_t p = outside(pg) ? 0 : pg;
      const uint32_t row = (g << pv.page_shift) + ((base + 16 * w) & in_page) + key;
      kraw[i] = *(const u32x4*)((const unsigned char*)pv.k + p * pv.page_stride + (size_t)row * HD + (ln % (HD / 16)) * 16);
      return;
    }
    static_assert(64 / CH <= CH && (Q8 ? 2 : 1) * KI * (64 / CH) == 16, "a wave's pieces are 16 keys, and a piece's permutation is that of piece 0, exclusive-or its first key");
    const int pg = __builtin_amdgcn_readlane(page, 4 * w), k0 = ln / CH, c0 = (ln % CH) ^ k0, ki = (w * KI + i) * (64 / CH);
    const bf16_t* src = (const bf16_t*)pv.k + (size_t)(outside(pg) ? 0 : pg) * pv.page_stride + (((size_t)g << pv.page_shift) + ((base + 16 * w) & in_page)) * HD;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + (uint32_t)((i * (64 / CH) + k0) * HD + (c0 ^ (ki & (CH - 1))) * 8)),
                                     (__attribute__((address_space(3))) void*)(uintptr_t)(ring + (uint32_t)(buf * TILE + (w * KI + i) * 512) * 2), 16, 0, 0);
  };
  // V: 4 keys of a page, DV dims a thread; keys behind the range's last are whatever the page holds there
  vraw_t vraw[Q8 ? 4 : 1];
  vwide_t vr[4];
  const CT* vsrc = nullptr;
  auto aim_v = [&](int ln, int base, int page) {
    if constexpr (Q8) {
      const size_t sc = (size_t)(outside(page) ? 0 : page) * pv.scale_stride + (uint32_t)((g << pv.page_shift) + ((base + 4 * (ln & 15)) & in_page));
      kscale = *(const uint32_t*)(pv.ks + sc);
      vscale = *(const uint32_t*)(pv.vs + sc);
    }
    vsrc = (const CT*)pv.v + (size_t)(outside(page) ? 0 : page) * pv.page_stride +
           (uint32_t)(((g << pv.page_shift) + ((base + 4 * (ln & 15)) & in_page)) * HD + (w * 4 + (ln >> 4)) * DV);
  };
  auto load_v = [&](int m) {
    if constexpr (Q8) vraw[m] = *(const vraw_t*)(vsrc + m * HD);
    else vr[m] = *(const vwide_t*)(vsrc + m * HD);
  };
  // 8-bit pools: what has been loaded, as bf16: the values in registers, the keys in LDS, as the direct loads of bf16 keys leave them
  auto widen = [&](int ln, int buf) {
    if constexpr (Q8) {
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const int key = 16 * w + (i * 64 + ln) / (HD / 16), c = 2 * (ln % (HD / 16));
        const float sk = e8m0_scale(((uint32_t)__shfl((int)kscale, key >> 2, 64) >> (8 * (key & 3))) & 0xFFu);
        const uint32_t at = ring + (uint32_t)(buf * TILE + key * HD) * 2;
        // (a key's eight lanes write chunks of which those 128 bytes apart share banks; with half of the lanes beginning with their second one nothing does, but the swaps cost more: 361 us for 358, measured with half of the output's products)
        uint32_t x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[2 * e] = e4m3_pair<false>(kraw[i][e], sk); x[2 * e + 1] = e4m3_pair<true>(kraw[i][e], sk); }
        *(lds_u32x4*)(uintptr_t)(at + ((c ^ (key & (CH - 1))) << 4)) = u32x4{x[0], x[1], x[2], x[3]};
        *(lds_u32x4*)(uintptr_t)(at + (((c + 1) ^ (key & (CH - 1))) << 4)) = u32x4{x[4], x[5], x[6], x[7]};
      }
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const float sv = e8m0_scale((vscale >> (8 * m)) & 0xFFu);
#pragma unroll
        for (int u = 0; u < VR; ++u) { vr[m][2 * u] = e4m3_pair<false>(vraw[m][u], sv); vr[m][2 * u + 1] = e4m3_pair<true>(vraw[m][u], sv); }
      }
    }
  };
  // values of pages outside the pool and of keys behind the last become 0; so do those from poison_s on that are not finite
  auto needs_clean = [&](int base, int page, bool drop) { return drop || base + KT > ke || __any(outside(page)); };
  auto clean_v = [&](int base, int page, bool drop) {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int key = base + 4 * (lane & 15) + m;
      if (outside(page) || key >= ke) {
#pragma unroll
        for (int u = 0; u < DV / 2; ++u) vr[m][u] = 0u;
      } else if (drop && key >= poison_s) {
#pragma unroll
        for (int u = 0; u < DV / 2; ++u)
          vr[m][u] = ((vr[m][u] & 0x7F80u) == 0x7F80u ? 0u : vr[m][u] & 0xFFFFu) | ((vr[m][u] & 0x7F800000u) == 0x7F800000u ? 0u : vr[m][u] & 0xFFFF0000u);
      }
    }
  };
  // A V^T row is a dim; 16 keys' groups of 4 lie in it in the order 0, 2, 1, 3, so that the two groups a lane of the product needs are one 16-byte slot; slots
  // permuted by the dim's pair, which for pair u of a thread is that of pair 0, exclusive-or u
  static_assert((DV / 2 & (DV / 2 - 1)) == 0 && DV / 2 <= 8, "pairs of a thread: low bits of the permutation");
  auto store_v = [&](int ln, int buf) {
    const int kgp = ln & 15, dg = w * 4 + (ln >> 4);
    const uint32_t at = ring + (uint32_t)((2 + buf) * TILE + dg * DV * KT) * 2 + (((2 * (kgp >> 2) + (kgp & 1)) ^ ((dg * (DV / 2)) & 7)) << 4) + (((kgp >> 1) & 1) << 3);
#pragma unroll
    for (int u = 0; u < DV / 2; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const unsigned int s = h ? 0x07060302u : 0x05040100u;
        *(lds_u32x2*)(uintptr_t)((at ^ (u << 4)) + (2 * u + h) * KT * 2) = u32x2{__builtin_amdgcn_perm(vr[1][u], vr[0][u], s), __builtin_amdgcn_perm(vr[3][u], vr[2][u], s)};
      }
  };
  const int n_tiles = (ke - kb + KT - 1) / KT;
  int pages = load_pages(kb), pages_next = load_pages(kb + KT);
  if (tid == 0) poison_s = INT_MAX;

  // the lane's query vector: dims 16 t + 8 hi + 0..7; its rotary partner dims (i, i + HD/2) are the lane's own
  bf16x8_t qh[T], ql[T];
  {
    float x[T][8];
    const float* src = qkv + (size_t)qkv_row * ld + (size_t)head * HD + 8 * hi;
    float ss = 0.f;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const f32x4 a = *(const f32x4*)(src + 16 * t), c = *(const f32x4*)(src + 16 * t + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[t][e] = a[e]; x[t][4 + e] = c[e]; }
    }
    // gains and angles are asked for together with the row, in front of the keys: one latency instead of three (a microsecond of a layer's 57, 64 rows of 32/8 heads behind 16384 shared tokens)
    f32x4 turn[T / 2][4];
    u32x4 gains[T];
    if (q_gain) {
#pragma unroll
      for (int t = 0; t < T; ++t) gains[t] = *(const u32x4*)(q_gain + 16 * t + 8 * hi);
    }
    if (rope_tab) {
      const f32x4* rp = (const f32x4*)(rope_tab + (size_t)rope_pos * (HD / 2) + 8 * hi);
#pragma unroll
      for (int t = 0; t < T / 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) turn[t][e] = rp[8 * t + e];
    }
#pragma unroll
    for (int i = 0; i < KI; ++i) load_k(lane, kb, pages, 0, i);
    aim_v(lane, kb, pages);
#pragma unroll
    for (int m = 0; m < 4; ++m) load_v(m);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += x[t][e] * x[t][e];
    ss = pair_sum<32>(ss);
    const float scale = rsqrtf((float)HD) * 1.4426950408889634f;
    if (q_gain) {
      const float rs = rsqrtf(ss / (float)HD + eps);
#pragma unroll
      for (int t = 0; t < T; ++t) {
        float gn[8];
        Elem<bf16_t>::unpack(gains[t], gn);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[t][e] *= rs * gn[e];
      }
    }
    if (rope_tab) {
#pragma unroll
      for (int t = 0; t < T / 2; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 cs = make_float2(turn[t][e / 2][2 * (e & 1)], turn[t][e / 2][2 * (e & 1) + 1]);
          const float a = x[t][e], b = x[t + T / 2][e];
          x[t][e] = a * cs.x - b * cs.y;
          x[t + T / 2][e] = b * cs.x + a * cs.y;
        }
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      uint32_t h4[4], l4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = x[t][2 * e] * scale, b = x[t][2 * e + 1] * scale;
        h4[e] = pack_bf16x2(a, b);
        l4[e] = pack_bf16x2(a - __uint_as_float(h4[e] << 16), b - __uint_as_float(h4[e] & 0xFFFF0000u));
      }
      qh[t] = __builtin_bit_cast(bf16x8_t, u32x4{h4[0], h4[1], h4[2], h4[3]});
      ql[t] = __builtin_bit_cast(bf16x8_t, u32x4{l4[0], l4[1], l4[2], l4[3]});
    }
  }
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  __syncthreads();
  // values at positions that some row of the block does not see, 16 bytes each: is one of them not finite?
  for (int c = tid; c < (ke - max(it.pos0 + 1, kb)) * CH; c += NT) {
    const int key = max(it.pos0 + 1, kb) + c / CH, page = trow[key >> pv.page_shift];
    if (outside(page)) continue;
    bool bad = false;
    const size_t row = ((size_t)g << pv.page_shift) + (key & in_page);
    if constexpr (Q8) {
      const uint2 codes = *(const uint2*)((const unsigned char*)pv.v + (size_t)page * pv.page_stride + row * HD + c % CH * 8);
      const float sv = e8m0_scale(pv.vs[(size_t)page * pv.scale_stride + row]);
      const uint32_t v[4] = {e4m3_pair<false>(codes.x, sv), e4m3_pair<true>(codes.x, sv), e4m3_pair<false>(codes.y, sv), e4m3_pair<true>(codes.y, sv)};
#pragma unroll
      for (int u = 0; u < 4; ++u) bad |= (v[u] & 0x7F80u) == 0x7F80u || (v[u] & 0x7F800000u) == 0x7F800000u;
    } else {
      const u32x4 v = *(const u32x4*)((const bf16_t*)pv.v + (size_t)page * pv.page_stride + row * HD + c % CH * 8);
#pragma unroll
      for (int u = 0; u < 4; ++u) bad |= (v[u] & 0x7F80u) == 0x7F80u || (v[u] & 0x7F800000u) == 0x7F800000u;
    }
    if (bad) atomicMin(&poison_s, key);
  }
  __syncthreads();
  const int poison = __builtin_amdgcn_readfirstlane(poison_s);
  const bool drop = poison != INT_MAX;
  widen(lane, 0);
  if (needs_clean(kb, pages, drop)) clean_v(kb, pages, drop);
  store_v(lane, 0);
  __syncthreads();

  for (int tl = 0; tl < n_tiles; ++tl) {
    const int buf = tl & 1, base = kb + tl * KT, ahead = base + KT;
    const bool more = tl + 1 < n_tiles;
    const unsigned long long missing = __ballot(outside(pages));
    const int pages_after = more ? load_pages(ahead + KT) : 0;
    // Fragment addresses: chunk 2 t + hi of a K row and slot 2 q + hi of a V^T row, permuted, differ from chunk and slot hi by an exclusive or
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const uint32_t ko = ring + (uint32_t)(buf * TILE * 2) + (ln & 31) * (HD * 2) + (((ln >> 5) ^ (ln & (CH - 1))) << 4);
    const uint32_t vo = ring + (uint32_t)((2 + buf) * TILE * 2) + (ln & 31) * (KT * 2) + (((ln >> 5) ^ ((ln >> 1) & 7)) << 4);
    auto read_k = [&](int k, int t) { return __builtin_bit_cast(bf16x8_t, *(const lds_u32x4*)(uintptr_t)((ko ^ (t << 5)) + k * 32 * HD * 2)); };
    auto read_v = [&](int q, int t) { return __builtin_bit_cast(bf16x8_t, *(const lds_u32x4*)(uintptr_t)((vo ^ (q << 5)) + t * 32 * KT * 2)); };
    if (more) aim_v(ln, ahead, pages_next);
    // scores (in units of log2) of keys base + 32 k + 8 (e / 4) + 4 hi + e % 4 for the lane's query
    f32x16 s[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[k][e] = 0.f;
    bf16x8_t kf[2][2];
    kf[0][0] = read_k(0, 0);
    kf[0][1] = read_k(1, 0);
    auto scores = [&](auto more_c) {
      constexpr int LD = decltype(more_c)::value ? KI + 4 : 0;          // loads of the next tile, shared out over the steps
#pragma unroll
      for (int t = 0; t < T; ++t) {
        if (t + 1 < T) {
          kf[(t + 1) & 1][0] = read_k(0, t + 1);
          kf[(t + 1) & 1][1] = read_k(1, t + 1);
        }
        s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t & 1][0], ql[t], s[0], 0, 0, 0);
        s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t & 1][1], ql[t], s[1], 0, 0, 0);
#pragma unroll
        for (int z = t * LD / T; z < (t + 1) * LD / T; ++z) {
          if (z < KI) load_k(ln, ahead, pages_next, buf ^ 1, z);
          else load_v(z - KI);
        }
        s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t & 1][0], qh[t], s[0], 0, 0, 0);
        s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t & 1][1], qh[t], s[1], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (more) scores(std::integral_constant<bool, true>());
    else scores(std::integral_constant<bool, false>());
    bf16x8_t vf[2];
    vf[0] = read_v(0, 0);
    if (base + KT > it.pos0 + 1) {      // keys beyond some row's position in this tile
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (base + 32 * k + 8 * (e >> 2) + 4 * hi + (e & 3) > my_pos) s[k][e] = -INFINITY;
    }
    if (missing) {                      // pages outside the pool: bit 8 k + 2 (e / 4) + hi is the group of 4 keys
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((missing >> (8 * k + 2 * (e >> 2) + hi)) & 1) s[k][e] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[0][e]);
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[1][e]);
    mx = pair_max<32>(mx);
    const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
    if (__any(m_new > m_run)) {
      const float f = __builtin_amdgcn_exp2f(m_run - m_use);
      l_run *= f;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] *= f;
      m_run = m_new;
    }
    // the 8 probabilities of a contraction step q in bf16 parts, pair j of them in as many pieces
    uint32_t pp[2][PARTS][4];
    auto piece = [&](int q, int j, int z) {
      const int e = 8 * (q & 1) + 2 * j;
      const float a = s[q >> 1][e], d = s[q >> 1][e + 1];
      if (z == 0) {
        s[q >> 1][e] = __builtin_amdgcn_exp2f(a - m_use);
        s[q >> 1][e + 1] = __builtin_amdgcn_exp2f(d - m_use);
      } else if (z == 2) {
        paged_split3(a, d, pp[q & 1][0][j], pp[q & 1][1][j], pp[q & 1][PARTS - 1][j]);
      } else {
        l_run += a;
        l_run += d;
        if (PARTS == 3) return;
        const uint32_t h = pack_bf16x2(a, d);
        pp[q & 1][0][j] = h;
        pp[q & 1][1][j] = pack_bf16x2(a - __uint_as_float(h << 16), d - __uint_as_float(h & 0xFFFF0000u));
      }
    };
    constexpr int PG = 4 / DT;          // pairs of the next step beside a V fragment's products
#pragma unroll
    for (int z = 0; z < PARTS; ++z)
#pragma unroll
      for (int j = 0; j < 4; ++j) piece(0, j, z);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const int n = q * DT + t;
        if (n + 1 < 4 * DT) vf[(n + 1) & 1] = read_v((n + 1) / DT, (n + 1) % DT);
#pragma unroll
        for (int z = 0; z < PARTS; ++z) {
          const uint32_t* f = pp[q & 1][PARTS - 1 - z];
          acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[n & 1], __builtin_bit_cast(bf16x8_t, u32x4{f[0], f[1], f[2], f[3]}), acc[t], 0, 0, 0);
          if (q < 3) {
#pragma unroll
            for (int j = 0; j < PG; ++j) piece(q + 1, t * PG + j, z);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (more) {
      widen(ln, buf ^ 1);
      if (needs_clean(ahead, pages_next, drop)) clean_v(ahead, pages_next, drop);
      store_v(ln, buf ^ 1);
    }
    pages = pages_next;
    pages_next = pages_after;
    __builtin_amdgcn_s_waitcnt(7 << 4);      // vmcnt(0) lgkmcnt(0): this wave's share of the next tile has landed
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  l_run = pair_sum<32>(l_run);
  // where the vector goes, worked out anew: kept through the loop it would be spilled
  int ln = lane;
  asm volatile("" : "+v"(ln));
  const int qo = 32 * w + (ln & 31), qor = pv.row_of(qo), ro = it.row0 + qor, ho = g * GQ + qo - qor * GQ, co = ho * HD + 4 * (ln >> 5);
  if (it.pos0 + qor >= poison) l_run = __uint_as_float(0x7FC00000u);
  if constexpr (SHARED) {
    if (qo < QV && it.unit >= 0) {
      float* sums = sp.sums(it.unit + qor, ho, HD) + 4 * (ln >> 5);
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) *(f32x4*)(sums + 32 * t + 8 * q) = f32x4{acc[t][4 * q], acc[t][4 * q + 1], acc[t][4 * q + 2], acc[t][4 * q + 3]};
      if (ln < 32) *(float2*)sp.weights(it.unit + qor, pv.nh, ho, HD) = make_float2(m_run, l_run);
    } else if (qo < QV) {
      const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
      const int to = sp.row(it, qor).x;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          paged_store4<bf16_t, PLANES>(po, to, co + 32 * t + 8 * q, f32x4{acc[t][4 * q] * inv, acc[t][4 * q + 1] * inv, acc[t][4 * q + 2] * inv, acc[t][4 * q + 3] * inv});
    }
  } else {
    constexpr size_t SLOT = (size_t)QVT * (HD + 2);
    if (it.n == 1) {
      if (qo < QV) {
        const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            paged_store4<bf16_t, PLANES>(po, it.first + ro, co + 32 * t + 8 * q, f32x4{acc[t][4 * q] * inv, acc[t][4 * q + 1] * inv, acc[t][4 * q + 2] * inv, acc[t][4 * q + 3] * inv});
      }
      return;
    }
    float* part = wk.part + ((size_t)(it.slot + it.split) * pv.nkv + g) * SLOT;
    if (qo < QV) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) *(f32x4*)(part + (size_t)qo * HD + 32 * t + 8 * q + 4 * (ln >> 5)) = f32x4{acc[t][4 * q], acc[t][4 * q + 1], acc[t][4 * q + 2], acc[t][4 * q + 3]};
      if (ln < 32) *(float2*)(part + (size_t)QVT * HD + 2 * qo) = make_float2(m_run, l_run);
    }
  }
}

template <typename CT, int HD, bool PLANES>
__device__ __forceinline__ void paged_attention_tall(int y, const int* __restrict__ cu, const int* __restrict__ start, const float* __restrict__ qkv, long ld,
                                                     const bf16_t* __restrict__ q_gain, const float2* __restrict__ rope_tab, float eps, int max_new, int lo, const PagedOut& po,
                                                     const PagedView& pv, const PagedWork& wk) {
  PagedItem it;
  if (!paged_find<256, 64, false, true>(pv, cu, start, max_new, pv.gq, lo, INT_MAX, pv.rpb_tall, wk.shift, PAGED_KEYS_TALL, y, it)) return;
  paged_tall_item<CT, HD, PLANES, false>(it, blockIdx.x, threadIdx.x, qkv, ld, q_gain, rope_tab, eps, po, pv, wk, SharedParts{});
}

// Block of a KV head (x), through the grid's two other dimensions, which end at 65535 each
__device__ __forceinline__ int paged_block() { return blockIdx.z * gridDim.y + blockIdx.y; }

template <typename CT, int HD, bool PLANES>
__global__ void __launch_bounds__(64 * PAGED_WAVES, sizeof(CT) == 2 ? 4 : 2) paged_attention_few_mfma_kernel(
    const int* __restrict__ cu, const int* __restrict__ start, const float* __restrict__ qkv, long ld, const typename PagedWide<CT>::type* __restrict__ q_gain, const float2* __restrict__ rope_tab, float eps,
    int max_new, int hi, PagedOut po, PagedView pv, PagedWork wk) {
  paged_attention_few<CT, HD, PLANES>(paged_block(), cu, start, qkv, ld, q_gain, rope_tab, eps, max_new, hi, po, pv, wk);
}

// Both kinds of requests in one launch, the longer blocks first: a chunk's leave the memory to the single tokens' (316 rows of a chunk and 14 tokens, 14/2 heads of 64: 17.5 us; when
// both ways stood side by side one launch after the other took 28, and where no single token was in the batch their launch 4.8)
template <typename CT, int HD, bool PLANES>
__global__ void __launch_bounds__(256, 2) paged_attention_both_mfma_kernel(const int* __restrict__ cu, const int* __restrict__ start, const float* __restrict__ qkv, long ld,
                                                                           const bf16_t* __restrict__ q_gain, const float2* __restrict__ rope_tab, float eps, int max_new, int border,
                                                                           int n_tall, PagedOut po, PagedView pv, PagedWork few, PagedWork tall) {
  static_assert(PAGED_WAVES == 4, "blocks of one size");
  const int y = paged_block();
  if (y < n_tall) paged_attention_tall<CT, HD, PLANES>(y, cu, start, qkv, ld, q_gain, rope_tab, eps, max_new, border, po, pv, tall);
  else paged_attention_few<CT, HD, PLANES>(y - n_tall, cu, start, qkv, ld, q_gain, rope_tab, eps, max_new, border, po, pv, few);
}

// The ranges of the tall kernel's groups joined: 64 KiB of partial results a group and range are too much for the block that ends last (64 rows behind
// 4096, 32/8 heads: 87 us by it against 41 with this launch when both were tried, 27 since; the launch is 4.8 of them, with nothing to join too).
template <int HD, bool PLANES>
__global__ void __launch_bounds__(256) paged_attention_merge_kernel(const int* __restrict__ cu, const int* __restrict__ start, int max_new, int lo, PagedOut po, PagedView pv,
                                                                    PagedWork wk) {
  constexpr int QVT = 128, NT = 256, T4 = HD / 4;
  constexpr size_t SLOT = (size_t)QVT * (HD + 2);
  const int g = blockIdx.x, GQ = pv.gq;
  PagedItem it;
  if (!paged_find<NT, 64, true>(pv, cu, start, max_new, GQ, lo, INT_MAX, pv.rpb_tall, wk.shift, PAGED_KEYS_TALL, blockIdx.z, it)) return;
  if (it.n < 2) return;      // the request's first range is all that the group sees: written
  const float* part = wk.part + ((size_t)it.slot * pv.nkv + g) * SLOT;
  const int d = (threadIdx.x % T4) * 4;
  for (int v = blockIdx.y * (NT / T4) + threadIdx.x / T4; v < it.r * GQ; v += gridDim.y * (NT / T4)) {      // one each, unless the groups are many
    PagedSum sum;
    sum.add_ranges<false>(part + (size_t)QVT * HD + 2 * v, part + (size_t)v * HD + d, (size_t)pv.nkv * SLOT, 0, it.n, 1);
    const int r = pv.row_of(v);
    paged_store4<bf16_t, PLANES>(po, it.first + it.row0 + r, (g * GQ + v - r * GQ) * HD + d, sum.result());
  }
}

}  // namespace dmtd
