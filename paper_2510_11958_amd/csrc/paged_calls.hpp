// The calls of the paged key/value cache (see include/dmtd.h): checks of their arguments, and the launches.
// Part of dmtd.hip: a failure's message goes where dmtd_last_error(NULL) finds it.
#pragma once
#include "attention_paged.hpp"
#include "attention_shared.hpp"

namespace {


int paged_fail(int code, const char* why) {
  g_create_error = why;
  return code;
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
bool page_size_ok(int p) { return p == 16 || p == 32 || p == 64 || p == 128 || p == 256; }
int log2_of(int p) { int s = 0; while ((1 << s) < p) ++s; return s; }

// Lets the blocks of a kernel have up to `most` bytes of dynamic LDS on the current device, once for each device (done: the kernel's own)
template <typename K>
hipError_t lds_room(K kern, size_t bytes, size_t most, bool (&done)[kMaxDevices]) {
  if (bytes <= 48 * 1024) return hipSuccess;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess || dev < 0 || dev >= kMaxDevices || done[dev]) return e;
  e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
  done[dev] = e == hipSuccess;
  return e;
}
// A grid of `blocks` blocks for each of nkv KV heads (paged_block)
dim3 paged_grid(int nkv, int blocks) {
  const int z = (blocks + 65534) / 65535;
  return dim3(nkv, (blocks + z - 1) / z, z);
}

// A launch goes to the device that is current; on a stream of another one it would fail or, worse, read that one's addresses here
int check_stream_device(hipStream_t s) {
  if (!s) return DMTD_OK;
  int cur = 0;
  hipDevice_t dev = 0;
  hipError_t e = hipGetDevice(&cur);
  if (e == hipSuccess) e = hipStreamGetDevice(s, &dev);
  if (e != hipSuccess) return paged_fail(DMTD_EHIP, hipGetErrorString(e));
  if ((int)dev != cur) return paged_fail(DMTD_EINVAL, "the stream belongs to another device than the current one");
  return DMTD_OK;
}

int paged_done() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DMTD_OK : paged_fail(DMTD_EHIP, hipGetErrorString(e));
}

int check_table(int n_req, int max_pages, int n_pages, int page_size) {
  if (!page_size_ok(page_size)) return paged_fail(DMTD_EINVAL, "page_size must be 16, 32, 64, 128 or 256");
  if (n_req < 1 || n_req > kPagedMaxRequests) return paged_fail(DMTD_EINVAL, "n_req must be in [1, 8192]");
  if (max_pages < 1 || (long)max_pages * page_size > (1L << 30)) return paged_fail(DMTD_EINVAL, "max_pages must be >= 1 and max_pages * page_size <= 2^30");
  if (n_pages < 1 || n_pages > (1 << 30)) return paged_fail(DMTD_EINVAL, "n_pages must be in [1, 2^30]");
  return DMTD_OK;
}

int check_cache(const dmtd_paged_cache* c) {
  if (!c) return paged_fail(DMTD_EINVAL, "null cache");
  const int rc = check_table(c->n_req, c->max_pages, c->n_pages, c->page_size);
  if (rc != DMTD_OK) return rc;
  const bool q8 = c->dtype == DMTD_DTYPE_E4M3;
  if (c->dtype != DMTD_DTYPE_F32 && c->dtype != DMTD_DTYPE_BF16 && !q8) return paged_fail(DMTD_EINVAL, "unknown dtype");
  if (c->head_dim != 64 && c->head_dim != 128) return paged_fail(DMTD_EINVAL, "head_dim must be 64 or 128");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > QV_MAX)
    return paged_fail(DMTD_EINVAL, "n_q_heads must be a multiple of n_kv_heads (at most 1024), at most 16 times as many");
  if (c->max_rows < 1 || c->max_rows > (1 << 24) || (long)c->max_rows * c->n_kv_heads > (1L << 27))
    return paged_fail(DMTD_EINVAL, "max_rows must be in [1, 2^24], and at most 2^27 with the KV heads");
  if (!c->k || !c->v || !c->block_table) return paged_fail(DMTD_EINVAL, "null cache pointer");
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->block_table, 4)) return paged_fail(DMTD_EINVAL, "k and v must be 16-byte aligned");
  const long one = (long)c->n_kv_heads * c->page_size * c->head_dim;
  if (c->page_stride != 0 && (c->page_stride < one || c->page_stride % (q8 ? 16 : 8))) return paged_fail(DMTD_EINVAL, "page_stride must be 0 or a multiple of 8 (e4m3: 16) that holds a page");
  if (!q8) return DMTD_OK;      // (callers of the other types may not know of the fields behind max_rows)
  if (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16)) return paged_fail(DMTD_EINVAL, "an e4m3 cache needs 16-byte aligned k_scale and v_scale");
  const long scales = (long)c->n_kv_heads * c->page_size;
  if (c->scale_stride != 0 && (c->scale_stride < scales || c->scale_stride % 16)) return paged_fail(DMTD_EINVAL, "scale_stride must be 0 or a multiple of 16 that holds a page's scales");
  return DMTD_OK;
}

// qkv rows of at least `cols` values, the norm's gain and the rotary table
int check_rows(const float* qkv, int64_t ld, int64_t cols, const void* gain, float eps, const float* rope, int32_t rope_len) {
  if (!qkv || !aligned(qkv, 16)) return paged_fail(DMTD_EINVAL, "qkv must be a 16-byte aligned pointer");
  if (ld < cols || ld % 4 || ld > (1 << 24)) return paged_fail(DMTD_EINVAL, "ld must be a multiple of 4 that holds a row");
  if (gain && !aligned(gain, 16)) return paged_fail(DMTD_EINVAL, "a norm's gain must be 16-byte aligned");
  if (gain && !(eps >= 0.f && eps < 1e30f)) return paged_fail(DMTD_EINVAL, "eps must be finite and not negative");
  if (rope && (!aligned(rope, 16) || rope_len < 1)) return paged_fail(DMTD_EINVAL, "the rotary table must be 16-byte aligned and hold a position");
  return DMTD_OK;
}

PagedView paged_view(const dmtd_paged_cache* c, const float* rope, int32_t rope_len) {
  PagedView v{};
  v.k = c->k; v.v = c->v; v.table = c->block_table;
  v.page_stride = c->page_stride ? c->page_stride : (long)c->n_kv_heads * c->page_size * c->head_dim;
  if (c->dtype == DMTD_DTYPE_E4M3) {
    v.ks = (unsigned char*)c->k_scale; v.vs = (unsigned char*)c->v_scale;
    v.scale_stride = c->scale_stride ? c->scale_stride : (long)c->n_kv_heads * c->page_size;
  }
  v.n_pages = c->n_pages; v.page_shift = log2_of(c->page_size); v.n_req = c->n_req; v.max_pages = c->max_pages;
  v.nh = c->n_q_heads; v.nkv = c->n_kv_heads; v.max_rows = c->max_rows;
  v.limit = c->max_pages * c->page_size;
  v.gq = v.nh / v.nkv; v.gq_mul = (1 << 16) / v.gq + 1; v.rpb_few = 16 / v.gq; v.rpb_tall = 128 / v.gq;
  if (rope && rope_len < v.limit) v.limit = rope_len;
  return v;
}

// Rows up to which the bookkeeping is one block's
constexpr int kTableRows = 2048;

template <typename CT>
void launch_paged_append(const PagedView& v, int head_dim, const float* qkv, long ld, const int* cu, const int* row_pos, const int64_t* slots, const void* gain,
                         float eps, const float* rope, hipStream_t s) {
  const dim3 grid((unsigned)(((long)v.max_rows * v.nkv + 15) / 16));
  if (head_dim == 128)
    hipLaunchKernelGGL((paged_append_kernel<CT, 128>), grid, dim3(256), 0, s, qkv, ld, cu, row_pos, (const long long*)slots, (const typename PagedWide<CT>::type*)gain, (const float2*)rope, eps, v);
  else
    hipLaunchKernelGGL((paged_append_kernel<CT, 64>), grid, dim3(256), 0, s, qkv, ld, cu, row_pos, (const long long*)slots, (const typename PagedWide<CT>::type*)gain, (const float2*)rope, eps, v);
}

template <typename CT>
void launch_paged_read(const PagedView& v, int head_dim, const int64_t* slots, int n, void* k_out, void* v_out, long ldo, hipStream_t s) {
  typedef typename PagedWide<CT>::type GT;
  const dim3 grid((unsigned)(((long)n * v.nkv + 15) / 16));
  if (head_dim == 128) hipLaunchKernelGGL((paged_read_kernel<CT, 128>), grid, dim3(256), 0, s, (const long long*)slots, n, (GT*)k_out, (GT*)v_out, ldo, v);
  else hipLaunchKernelGGL((paged_read_kernel<CT, 64>), grid, dim3(256), 0, s, (const long long*)slots, n, (GT*)k_out, (GT*)v_out, ldo, v);
}

// How an attention call is laid out: blocks per KV head of either kernel (0: no launch), groups that the merge looks at, log2 of those that the key ranges are chosen
// for, and the workspace: the counts of the few-rows groups with several ranges, their partial results, the tall groups' (paged_find).
struct PagedPlan { int few, tall, merge, few_shift, tall_shift; size_t count_bytes, few_bytes, tall_bytes; };
// The counts' room is the same for all caches, so that nothing else is ever written there and caches of different layouts may use one workspace in turn: fewer than
// 2^few_shift groups of each KV head count, which is at most 512 counts in all (1024 KV heads: none).
constexpr size_t PAGED_COUNT_BYTES = 4096;
int floor_log2(int v) { int s = 0; while ((2 << s) <= v) ++s; return s; }
PagedPlan paged_plan(const dmtd_paged_cache* c, int max_new) {
  PagedPlan p{};
  const int GQ = c->n_q_heads / c->n_kv_heads;
  const long limit = (long)c->max_pages * c->page_size;
  const bool bf16 = c->dtype != DMTD_DTYPE_F32;      // bf16 products
  p.few_shift = floor_log2(std::max((bf16 ? PAGED_SLOTS_FEW : PAGED_SLOTS_FP32) / c->n_kv_heads, 1));
  p.tall_shift = floor_log2(std::max(PAGED_SLOTS_TALL / c->n_kv_heads, 1));
  auto blocks = [&](long groups, int shift, int min_keys) { return (int)std::min((1L << shift) + groups, groups * ((limit + min_keys - 1) / min_keys)); };
  // a request with n rows is in ceil(n / rows of a group) groups
  const long few_rows = std::min<long>(c->max_rows, max_new), all = std::min(c->n_req, c->max_rows);
  const int rpb_few = 16 / GQ, rpb_tall = 128 / GQ, tall_from = PAGED_FEW / GQ + 1;
  long few = std::min<long>(c->max_rows, all + c->max_rows / rpb_few);
  if (bf16) few = std::min<long>(few, (long)c->n_req * ((tall_from - 1 + rpb_few - 1) / rpb_few));
  p.few = blocks(few, p.few_shift, PAGED_KEYS_FEW);
  p.few_bytes = align_up(((size_t)16 * (c->head_dim + 2) * 4 << p.few_shift) * 2 * c->n_kv_heads, 256);
  p.count_bytes = PAGED_COUNT_BYTES;
  if (bf16 && few_rows >= tall_from) {
    const long groups = std::min<long>(c->n_req, c->max_rows / tall_from) + c->max_rows / rpb_tall;
    p.tall = blocks(groups, p.tall_shift, PAGED_KEYS_TALL);
    p.merge = (int)std::min(groups, 1L << p.tall_shift);
    p.tall_bytes = ((size_t)128 * (c->head_dim + 2) * 4 << p.tall_shift) * 2 * c->n_kv_heads;
  }
  return p;
}

struct PagedCall {
  const float* qkv; long ld;
  const int *start, *cu;
  int max_new;
  const void* gain;
  float eps;
  const float* rope;
  char* ws;
  hipStream_t stream;
};

template <typename CT, int HD, bool PLANES>
hipError_t launch_paged_attention_t(const PagedView& v, const PagedPlan& p, const PagedCall& a, const PagedOut& out) {
  const int GQ = v.nh / v.nkv;
  typedef typename PagedWide<CT>::type GT;
  constexpr bool BF = sizeof(GT) == 2;
  // The two kinds of requests have partial results of their own: they may be under way at the same time
  const PagedWork few{p.few_shift, (int*)a.ws, (float*)(a.ws + p.count_bytes)}, tall{p.tall_shift, nullptr, (float*)(a.ws + p.count_bytes + p.few_bytes)};
  // the queries' parts, then the waves' results, then what the join exchanges
  const int qv_max = std::min(16 / GQ, a.max_new) * GQ;
  const size_t few_lds = std::max({(size_t)PAGED_WAVES * qv_max * HD * 4, (size_t)16 * (BF ? 2 * (HD + ATT_QPAD) * 2 : (HD + 4) * 4), (size_t)2 * 64 * PAGED_WAVES * 16});
  if constexpr (BF) {
    if (p.tall > 0) {
      auto kern = paged_attention_both_mfma_kernel<CT, HD, PLANES>;
      const size_t lds = std::max((size_t)4 * 64 * HD * 2 + 1024, few_lds);      // (the rings start at a multiple of 1 KiB)
      static bool big_lds[kMaxDevices];
      const hipError_t e = lds_room(kern, lds, (size_t)4 * 64 * 128 * 2 + 1024, big_lds);
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(kern, paged_grid(v.nkv, p.tall + p.few), dim3(256), lds, a.stream, a.cu, a.start, a.qkv, a.ld, (const bf16_t*)a.gain, (const float2*)a.rope, a.eps, a.max_new, PAGED_FEW,
                         p.tall, out, v, few, tall);
      // a vector per thread as long as that makes at most 1024 blocks, most of which have nothing to do
      const int merge_blocks = std::min(HD / 8, std::max(HD / 32, 1024 / (v.nkv * p.merge)));
      hipLaunchKernelGGL((paged_attention_merge_kernel<HD, PLANES>), dim3(v.nkv, merge_blocks, p.merge), dim3(256), 0, a.stream, a.cu, a.start, a.max_new, PAGED_FEW, out, v, tall);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((paged_attention_few_mfma_kernel<CT, HD, PLANES>), paged_grid(v.nkv, p.few), dim3(64 * PAGED_WAVES), few_lds, a.stream, a.cu, a.start, a.qkv, a.ld, (const GT*)a.gain,
                     (const float2*)a.rope, a.eps, a.max_new, BF ? PAGED_FEW : INT_MAX, out, v, few);
  return hipGetLastError();
}

// out.lo not null (bf16): the two planes that the projections read, instead of rows of the cache's type
hipError_t launch_paged_attention(const dmtd_paged_cache* c, const PagedView& v, const PagedCall& a, const PagedOut& out) {
  const PagedPlan p = paged_plan(c, a.max_new);
  if (c->dtype == DMTD_DTYPE_BF16 && out.lo) return c->head_dim == 128 ? launch_paged_attention_t<bf16_t, 128, true>(v, p, a, out) : launch_paged_attention_t<bf16_t, 64, true>(v, p, a, out);
  if (c->dtype == DMTD_DTYPE_BF16) return c->head_dim == 128 ? launch_paged_attention_t<bf16_t, 128, false>(v, p, a, out) : launch_paged_attention_t<bf16_t, 64, false>(v, p, a, out);
  if (c->dtype == DMTD_DTYPE_E4M3) return c->head_dim == 128 ? launch_paged_attention_t<e4m3_t, 128, false>(v, p, a, out) : launch_paged_attention_t<e4m3_t, 64, false>(v, p, a, out);
  return c->head_dim == 128 ? launch_paged_attention_t<float, 128, false>(v, p, a, out) : launch_paged_attention_t<float, 64, false>(v, p, a, out);
}

// ---- shared prefixes ----

// How a step with shared prefixes is laid out: log2 of the blocks per KV head that the key ranges are chosen for, the most items there can be, a unit of partial results, and the sizes.
struct SharedPlanSizes { int few_shift, tall_shift, few_max, few_keys; long items, units, unit_floats; size_t list, recs, scratch, plan_bytes; };
SharedPlanSizes shared_sizes(const dmtd_paged_cache* c, int n_groups) {
  SharedPlanSizes z{};
  const int GQ = c->n_q_heads / c->n_kv_heads, rpb_few = 16 / GQ, rpb_tall = 128 / GQ;
  const bool bf16 = c->dtype != DMTD_DTYPE_F32;
  z.few_shift = floor_log2(std::max(SHARE_SLOTS_FEW / c->n_kv_heads, 1));
  z.tall_shift = floor_log2(std::max(SHARE_SLOTS_TALL / c->n_kv_heads, 1));
  z.few_max = bf16 ? SHARE_FEW : INT_MAX;
  z.few_keys = bf16 ? PAGED_KEYS_FEW : SHARE_KEYS_FP32;
  // entries are the requests and the groups of two and more; one of n rows has ceil(n / rows of a tile) tiles, and the ranges of all come to a tile's first and at most 2^shift more of either kind (twice that of tall ones)
  const long R = c->max_rows, reqs = std::min<long>(c->n_req, R);
  z.items = reqs + std::min<long>(n_groups, reqs / 2) + 2 * (R / rpb_few) + (1L << z.few_shift) + (2L << z.tall_shift);
  z.units = 2 * R + ((long)rpb_few << z.few_shift) + ((long)rpb_tall << (z.tall_shift + 1));
  z.unit_floats = (long)c->n_q_heads * c->head_dim + (2 * c->n_q_heads + 3) / 4 * 4;
  size_t off = SHARE_HEADER * 4 + (size_t)z.items * 32;
  auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes, 16); return o; };
  z.list = take((size_t)R * 8);
  z.recs = take((size_t)R * 32);
  z.scratch = take((size_t)ShareTables::ints(c->n_req, n_groups) * 4);
  z.plan_bytes = align_up(off, 256);
  return z;
}
SharePlan share_plan(const SharedPlanSizes& z, void* at) {
  char* p = (char*)at;
  return SharePlan{(int*)p, (int4*)(p + SHARE_HEADER * 4), (int2*)(p + z.list), (int4*)(p + z.recs), (int*)(p + z.scratch)};
}
// What a plan is laid out for; the attention does nothing with a plan of another sign
int shared_sign(const dmtd_paged_cache* c, int n_groups, int positions) {
  uint32_t h = 2166136261u;
  for (int v : {c->n_req, c->max_pages, c->page_size, c->n_q_heads, c->n_kv_heads, c->head_dim, (int)(c->dtype == DMTD_DTYPE_F32), c->max_rows, n_groups, positions})
    for (int b = 0; b < 32; b += 8) h = (h ^ (((uint32_t)v >> b) & 0xFFu)) * 16777619u;
  return (int)(h | 1u);
}
int check_shared(const dmtd_paged_cache* c, const dmtd_shared_plan* p) {
  const int rc = check_cache(c);
  if (rc != DMTD_OK) return rc;
  if (!p) return paged_fail(DMTD_EINVAL, "null plan");
  if (p->n_groups < 1 || p->n_groups > kShareMaxGroups) return paged_fail(DMTD_EINVAL, "n_groups must be in [1, 8192]");
  if (p->positions < 0) return paged_fail(DMTD_EINVAL, "positions must not be negative");
  if (!p->plan || !aligned(p->plan, 256)) return paged_fail(DMTD_EINVAL, "the plan's memory must be 256-byte aligned");
  if (!p->workspace || !aligned(p->workspace, 256)) return paged_fail(DMTD_EINVAL, "workspace must be a 256-byte aligned pointer");
  if (p->plan_bytes < dmtd_shared_plan_bytes(c, p->n_groups)) return paged_fail(DMTD_ECAPACITY, "the plan's memory is too small");
  if (p->workspace_bytes < dmtd_shared_workspace_bytes(c)) return paged_fail(DMTD_ECAPACITY, "workspace too small");
  return DMTD_OK;
}

struct SharedCall {
  SharePlan plan;
  int sign;
  const float* qkv; long ld;
  const void* gain;
  float eps;
  const float* rope;
  hipStream_t stream;
};

template <typename CT, int HD>
hipError_t launch_shared_t(const PagedView& v, long items, const SharedCall& a, const PagedOut& out, const SharedParts& sp) {
  typedef typename PagedWide<CT>::type GT;
  constexpr bool BF = sizeof(GT) == 2;
  const size_t few_lds = (size_t)4 * 16 * (BF ? 2 * (HD + ATT_QPAD) * 2 : (HD + 4) * 4);      // the queries of each wave
  const long want = items * v.nkv;
  if (BF && (long)v.max_rows * v.gq > SHARE_FEW) {
    if constexpr (BF) {
      auto kern = paged_shared_mfma_kernel<CT, HD, true>;
      const size_t lds = std::max((size_t)4 * 64 * HD * 2 + 1024, few_lds);
      static bool big_lds[kMaxDevices];
      const hipError_t e = lds_room(kern, lds, (size_t)4 * 64 * 128 * 2 + 1024, big_lds);
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(kern, dim3((unsigned)std::min<long>(want, PAGED_RESIDENT_TALL)), dim3(256), lds, a.stream, a.plan, a.sign, (int)items, a.qkv, a.ld, (const GT*)a.gain, (const float2*)a.rope, a.eps, out, v, sp);
    }
  } else {
    constexpr int resident = 512;
    hipLaunchKernelGGL((paged_shared_mfma_kernel<CT, HD, false>), dim3((unsigned)std::min<long>((want + 3) / 4, resident)), dim3(256), few_lds, a.stream, a.plan, a.sign, (int)items, a.qkv, a.ld, (const GT*)a.gain,
                       (const float2*)a.rope, a.eps, out, v, sp);
  }
  const long waves = (long)v.max_rows * v.nh;
  hipLaunchKernelGGL((paged_shared_join_kernel<GT, HD>), dim3((unsigned)std::min<long>((waves + 3) / 4, 2048)), dim3(256), 0, a.stream, a.plan, a.sign, out, v, sp);
  return hipGetLastError();
}

}  // namespace

extern "C" {

int dmtd_page_tables(const dmtd_page_pool* p, const int32_t* start, const int32_t* rows, int32_t max_rows, int32_t* cu_rows, int32_t* row_pos,
                     int64_t* slots, int32_t* status, void* stream) {
  return dmtd_page_tables_shared(p, start, rows, nullptr, max_rows, cu_rows, row_pos, slots, status, stream);
}

int dmtd_page_tables_shared(const dmtd_page_pool* p, const int32_t* start, const int32_t* rows, const int32_t* shared, int32_t max_rows, int32_t* cu_rows,
                            int32_t* row_pos, int64_t* slots, int32_t* status, void* stream) {
  if (!p) return paged_fail(DMTD_EINVAL, "null pool");
  int rc = check_table(p->n_req, p->max_pages, p->n_pages, p->page_size);
  if (rc != DMTD_OK) return rc;
  if (!p->block_table || !p->held || !p->free_pages || !p->n_free || !start || !rows || !cu_rows || !row_pos || !slots || !status)
    return paged_fail(DMTD_EINVAL, "null pointer");
  for (const void* q : {(const void*)p->block_table, (const void*)p->held, (const void*)p->free_pages, (const void*)p->n_free, (const void*)start, (const void*)rows,
                        (const void*)shared, (const void*)cu_rows, (const void*)row_pos, (const void*)status})
    if (!aligned(q, 4)) return paged_fail(DMTD_EINVAL, "int32 arrays must be 4-byte aligned");
  if (!aligned(slots, 8)) return paged_fail(DMTD_EINVAL, "slots must be 8-byte aligned");
  if (max_rows < 1 || max_rows > (1 << 24)) return paged_fail(DMTD_EINVAL, "max_rows must be in [1, 2^24]");
  const hipStream_t s = (hipStream_t)stream;
  if ((rc = check_stream_device(s)) != DMTD_OK) return rc;
  const PageArgs a{p->block_table, p->held, p->free_pages, p->n_free, start, rows, shared, p->n_req, p->max_pages, p->n_pages, log2_of(p->page_size), max_rows, cu_rows, row_pos,
                   (long long*)slots, status};
  const size_t lds = (size_t)16 * p->n_req;          // of a block that moves pages
  static bool big_tables[kMaxDevices], big_moves[kMaxDevices];
  hipError_t e = hipSuccess;
  if (max_rows > kTableRows) {
    if ((e = lds_room(page_moves_kernel, lds, 16 * kPagedMaxRequests, big_moves)) != hipSuccess) return paged_fail(DMTD_EHIP, hipGetErrorString(e));
    hipLaunchKernelGGL(page_sums_kernel, dim3(1), dim3(1024), 0, s, a);
    hipLaunchKernelGGL(page_moves_kernel, dim3(64), dim3(256), lds, s, a);
    hipLaunchKernelGGL(page_rows_kernel, dim3((max_rows + 1023) / 1024 + 1), dim3(256), (size_t)4 * p->n_req, s, a);
  } else if (p->n_req <= 64 && max_rows <= 256) {
    hipLaunchKernelGGL(page_tables_kernel<64>, dim3(1), dim3(64), lds, s, a);
  } else if (p->n_req <= 256 && max_rows <= 1024) {
    hipLaunchKernelGGL(page_tables_kernel<256>, dim3(1), dim3(256), lds, s, a);
  } else {
    if ((e = lds_room(page_tables_kernel<1024>, lds, 16 * kPagedMaxRequests, big_tables)) != hipSuccess) return paged_fail(DMTD_EHIP, hipGetErrorString(e));
    hipLaunchKernelGGL(page_tables_kernel<1024>, dim3(1), dim3(1024), lds, s, a);
  }
  return paged_done();
}

int dmtd_paged_append(const dmtd_paged_cache* c, const float* qkv, int64_t ld, const int32_t* cu_rows, const int32_t* row_pos, const int64_t* slots,
                      const void* k_norm, float eps, const float* rope, int32_t rope_len, void* stream) {
  int rc = check_cache(c);
  if (rc == DMTD_OK) rc = check_rows(qkv, ld, (int64_t)(c->n_q_heads + 2 * c->n_kv_heads) * c->head_dim, k_norm, eps, rope, rope_len);
  if (rc != DMTD_OK) return rc;
  if (!cu_rows || !row_pos || !slots || !aligned(cu_rows, 4) || !aligned(row_pos, 4) || !aligned(slots, 8)) return paged_fail(DMTD_EINVAL, "bad row map pointer");
  const hipStream_t s = (hipStream_t)stream;
  if ((rc = check_stream_device(s)) != DMTD_OK) return rc;
  const PagedView v = paged_view(c, rope, rope_len);
  if (c->dtype == DMTD_DTYPE_BF16) launch_paged_append<bf16_t>(v, c->head_dim, qkv, ld, cu_rows, row_pos, slots, k_norm, eps, rope, s);
  else if (c->dtype == DMTD_DTYPE_E4M3) launch_paged_append<e4m3_t>(v, c->head_dim, qkv, ld, cu_rows, row_pos, slots, k_norm, eps, rope, s);
  else launch_paged_append<float>(v, c->head_dim, qkv, ld, cu_rows, row_pos, slots, k_norm, eps, rope, s);
  return paged_done();
}

int dmtd_paged_read(const dmtd_paged_cache* c, const int64_t* slots, int32_t n, void* k_out, void* v_out, int64_t ldo, void* stream) {
  int rc = check_cache(c);
  if (rc != DMTD_OK) return rc;
  if (n < 0 || (long)n * c->n_kv_heads > (1L << 27)) return paged_fail(DMTD_EINVAL, "n must not be negative, and at most 2^27 with the KV heads");
  if (!slots || !aligned(slots, 8)) return paged_fail(DMTD_EINVAL, "slots must be an 8-byte aligned pointer");
  if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return paged_fail(DMTD_EINVAL, "k_out and v_out must be 16-byte aligned pointers");
  if (ldo < (int64_t)c->n_kv_heads * c->head_dim || ldo % 8 || ldo > (1 << 24)) return paged_fail(DMTD_EINVAL, "ldo must be a multiple of 8 that holds a row");
  const hipStream_t s = (hipStream_t)stream;
  if ((rc = check_stream_device(s)) != DMTD_OK) return rc;
  if (n == 0) return DMTD_OK;
  const PagedView v = paged_view(c, nullptr, 0);
  if (c->dtype == DMTD_DTYPE_BF16) launch_paged_read<bf16_t>(v, c->head_dim, slots, n, k_out, v_out, (long)ldo, s);
  else if (c->dtype == DMTD_DTYPE_E4M3) launch_paged_read<e4m3_t>(v, c->head_dim, slots, n, k_out, v_out, (long)ldo, s);
  else launch_paged_read<float>(v, c->head_dim, slots, n, k_out, v_out, (long)ldo, s);
  return paged_done();
}

size_t dmtd_paged_workspace_bytes(const dmtd_paged_cache* c) {
  if (check_cache(c) != DMTD_OK) return 0;
  const PagedPlan p = paged_plan(c, c->max_rows);
  return p.count_bytes + p.few_bytes + p.tall_bytes;
}

int dmtd_paged_attention(const dmtd_paged_cache* c, const float* qkv, int64_t ld, const int32_t* start, const int32_t* cu_rows, int32_t max_new,
                         const void* q_norm, float eps, const float* rope, int32_t rope_len, void* out, int64_t ldo, void* workspace,
                         size_t workspace_bytes, void* stream) {
  int rc = check_cache(c);
  if (rc == DMTD_OK) rc = check_rows(qkv, ld, (int64_t)c->n_q_heads * c->head_dim, q_norm, eps, rope, rope_len);
  if (rc != DMTD_OK) return rc;
  if (!start || !cu_rows || !aligned(start, 4) || !aligned(cu_rows, 4)) return paged_fail(DMTD_EINVAL, "bad length pointer");
  if (max_new < 0 || max_new > c->max_rows) return paged_fail(DMTD_EINVAL, "max_new must be in [0, max_rows]");
  if (!out || !aligned(out, 16)) return paged_fail(DMTD_EINVAL, "out must be a 16-byte aligned pointer");
  if (ldo < (int64_t)c->n_q_heads * c->head_dim || ldo % 8 || ldo > (1 << 24)) return paged_fail(DMTD_EINVAL, "ldo must be a multiple of 8 that holds a row");
  if (!workspace || !aligned(workspace, 256)) return paged_fail(DMTD_EINVAL, "workspace must be a 256-byte aligned pointer");
  if (workspace_bytes < dmtd_paged_workspace_bytes(c)) return paged_fail(DMTD_ECAPACITY, "workspace too small");
  const hipStream_t s = (hipStream_t)stream;
  if ((rc = check_stream_device(s)) != DMTD_OK) return rc;
  const PagedView v = paged_view(c, rope, rope_len);
  if (max_new == 0) max_new = c->max_rows;
  const hipError_t e = launch_paged_attention(c, v, PagedCall{qkv, (long)ld, start, cu_rows, max_new, q_norm, eps, rope, (char*)workspace, s}, PagedOut{out, nullptr, (long)ldo, 0});
  return e == hipSuccess ? DMTD_OK : paged_fail(DMTD_EHIP, hipGetErrorString(e));
}

size_t dmtd_shared_plan_bytes(const dmtd_paged_cache* c, int32_t n_groups) {
  if (check_cache(c) != DMTD_OK) return 0;
  if (n_groups < 1 || n_groups > kShareMaxGroups) { paged_fail(DMTD_EINVAL, "n_groups must be in [1, 8192]"); return 0; }
  return shared_sizes(c, n_groups).plan_bytes;
}

size_t dmtd_shared_workspace_bytes(const dmtd_paged_cache* c) {
  if (check_cache(c) != DMTD_OK) return 0;
  const SharedPlanSizes z = shared_sizes(c, 1);
  return (size_t)z.units * z.unit_floats * 4;
}

int dmtd_shared_plan_build(const dmtd_paged_cache* c, const dmtd_shared_plan* p, const int32_t* start, const int32_t* cu_rows, const int32_t* group, const int32_t* prefix_pages,
                           void* stream) {
  int rc = check_shared(c, p);
  if (rc != DMTD_OK) return rc;
  for (const void* q : {(const void*)start, (const void*)cu_rows, (const void*)group, (const void*)prefix_pages})
    if (!q || !aligned(q, 4)) return paged_fail(DMTD_EINVAL, "start, cu_rows, group and prefix_pages must be 4-byte aligned pointers");
  const hipStream_t s = (hipStream_t)stream;
  if ((rc = check_stream_device(s)) != DMTD_OK) return rc;
  PagedView v = paged_view(c, nullptr, 0);
  if (p->positions && p->positions < v.limit) v.limit = p->positions;
  const SharedPlanSizes z = shared_sizes(c, p->n_groups);
  const ShareArgs a{start, cu_rows, group, prefix_pages, p->n_groups, z.few_shift, z.tall_shift, z.few_max, z.few_keys, shared_sign(c, p->n_groups, p->positions), share_plan(z, p->plan)};
  const size_t tables = (size_t)ShareTables::ints(c->n_req, p->n_groups) * 4;
  static bool big_tables[kMaxDevices], big_counts[kMaxDevices];
  const int most = std::max(c->n_req, p->n_groups);
  hipError_t e = hipSuccess;
  if (most <= 256 && c->max_rows <= 1024) {
    hipLaunchKernelGGL((share_plan_kernel<256, true>), dim3(1), dim3(256), tables, s, a, v);
  } else if (most <= SHARE_LDS_ENTRIES) {
    e = lds_room(share_plan_kernel<1024, true>, tables, (size_t)ShareTables::ints(SHARE_LDS_ENTRIES, SHARE_LDS_ENTRIES) * 4, big_tables);
    if (e == hipSuccess) hipLaunchKernelGGL((share_plan_kernel<1024, true>), dim3(1), dim3(1024), tables, s, a, v);
  } else {
    const size_t lds = (size_t)8 * p->n_groups;
    e = lds_room(share_plan_kernel<1024, false>, lds, (size_t)8 * kShareMaxGroups, big_counts);
    if (e == hipSuccess) hipLaunchKernelGGL((share_plan_kernel<1024, false>), dim3(1), dim3(1024), lds, s, a, v);
  }
  if (e != hipSuccess) return paged_fail(DMTD_EHIP, hipGetErrorString(e));
  return paged_done();
}

int dmtd_paged_attention_shared(const dmtd_paged_cache* c, const dmtd_shared_plan* p, const float* qkv, int64_t ld, const void* q_norm, float eps, const float* rope, int32_t rope_len,
                                void* out, int64_t ldo, void* stream) {
  int rc = check_shared(c, p);
  if (rc == DMTD_OK) rc = check_rows(qkv, ld, (int64_t)c->n_q_heads * c->head_dim, q_norm, eps, rope, rope_len);
  if (rc != DMTD_OK) return rc;
  if (!out || !aligned(out, 16)) return paged_fail(DMTD_EINVAL, "out must be a 16-byte aligned pointer");
  if (ldo < (int64_t)c->n_q_heads * c->head_dim || ldo % 8 || ldo > (1 << 24)) return paged_fail(DMTD_EINVAL, "ldo must be a multiple of 8 that holds a row");
  PagedView v = paged_view(c, nullptr, 0);
  if (p->positions && p->positions < v.limit) v.limit = p->positions;
  if (rope && rope_len < v.limit) return paged_fail(DMTD_EINVAL, "the rotary table is shorter than the positions that the plan is made for");
  const hipStream_t s = (hipStream_t)stream;
  if ((rc = check_stream_device(s)) != DMTD_OK) return rc;
  const SharedPlanSizes z = shared_sizes(c, p->n_groups);
  const SharePlan plan = share_plan(z, p->plan);
  const SharedCall a{plan, shared_sign(c, p->n_groups, p->positions), qkv, (long)ld, q_norm, eps, rope, s};
  const PagedOut to{out, nullptr, (long)ldo, 0};
  const SharedParts sp{plan.list, (float*)p->workspace, z.unit_floats};
  hipError_t e;
  if (c->dtype == DMTD_DTYPE_BF16) e = c->head_dim == 128 ? launch_shared_t<bf16_t, 128>(v, z.items, a, to, sp) : launch_shared_t<bf16_t, 64>(v, z.items, a, to, sp);
  else if (c->dtype == DMTD_DTYPE_E4M3) e = c->head_dim == 128 ? launch_shared_t<e4m3_t, 128>(v, z.items, a, to, sp) : launch_shared_t<e4m3_t, 64>(v, z.items, a, to, sp);
  else e = c->head_dim == 128 ? launch_shared_t<float, 128>(v, z.items, a, to, sp) : launch_shared_t<float, 64>(v, z.items, a, to, sp);
  return e == hipSuccess ? DMTD_OK : paged_fail(DMTD_EHIP, hipGetErrorString(e));
}

}  // extern "C"
