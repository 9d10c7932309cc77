// Steps of a context over requests that come and go (dmtd_paged_begin and the calls behind it; see include/dmtd.h): the context's caches serve as a pool of
// pages, and a step is one pass of the front layers over the rows that pass them and one of the late layers over the new tokens, rows of all
// requests behind one another.  Projections as in a prefill pass; append and attention are those of the paged cache (paged.hpp, attention_paged.hpp).
// Part of dmtd.hip.
#pragma once

namespace {

// Rows of a pass, behind one another, for the norm of the layer they enter: row idx[j] of src (idx null or negative: none) plus, where there is none or `add` says so (the
// literal reading of Eq. 4), the embedding of token tokens[j].
template <typename WT, bool PACK>
__global__ void __launch_bounds__(256) paged_rows_kernel(const float* __restrict__ src, const int* __restrict__ idx, const int* __restrict__ tokens, int add,
                                                         const WT* __restrict__ table, float* __restrict__ dst, int d, const bf16_t* __restrict__ gain,
                                                         bf16_t* __restrict__ xb, bf16_t* __restrict__ xb_lo, float* __restrict__ ssp, int blocked) {
  const int j = blockIdx.x, s = idx ? idx[j] : -1;
  const float* from = s >= 0 ? src + (size_t)s * d : nullptr;
  const WT* e = s < 0 || add ? table + (size_t)tokens[j] * d : nullptr;
  float* o = dst + (size_t)j * d;
  for (int k = threadIdx.x; k < d; k += blockDim.x) o[k] = (from ? from[k] : 0.f) + (e ? Elem<WT>::to_f32(e[k]) : 0.f);
  if (PACK) pack_row_for_norm(o, gain, d, blocked, j, xb, xb_lo, ssp + j);
}

// A row's token from its selection keys (see finish_step_kernel), which are cleared; one wave a row
__global__ void __launch_bounds__(64) paged_pick_kernel(unsigned long long* __restrict__ amax, int n_cells, int amax_ld, int* __restrict__ out) {
  const int b = blockIdx.x, lane = threadIdx.x;
  unsigned long long best = 0ull;
  if (lane < n_cells) {
    best = amax[(size_t)lane * amax_ld + b];
    amax[(size_t)lane * amax_ld + b] = 0ull;
  }
  best = wave_max_key(best);
  if (lane == 0) out[b] = argmax_key_index(best);
}

hipError_t paged_rows(dmtd_ctx* c, int n, const float* src, const int* idx, const int* tokens, bool add, Rows& R, int next_layer) {
  const dmtd_config& cf = c->cfg;
  if (c->packed)
    hipLaunchKernelGGL((paged_rows_kernel<bf16_t, true>), dim3(n), dim3(256), 0, c->stream, src, idx, tokens, add ? 1 : 0, (const bf16_t*)c->embed, R.h, cf.hidden,
                       (const bf16_t*)norm_gain_for_layer(c, next_layer), R.xb, R.xb_lo, R.ssp, blocked_rows(c, n));
  else
    hipLaunchKernelGGL((paged_rows_kernel<float, false>), dim3(n), dim3(256), 0, c->stream, src, idx, tokens, add ? 1 : 0, (const float*)c->embed, R.h, cf.hidden,
                       (const bf16_t*)nullptr, (bf16_t*)nullptr, (bf16_t*)nullptr, (float*)nullptr, 0);
  R.n_parts = 1;
  return hipGetLastError();
}

// The DEVICE memory of a context's paged steps, in bytes from its start
struct PagedLayout {
  int page, max_pages, n_pages, rows;
  static constexpr int kStatus = 4;      // ints at `status`: what the tables of either pass say (paged_tables), which the tokens follow that a step emits
  size_t table, held, free_pages, n_free, status, up, cu[2], pos[2], slots[2], attention, attention_bytes, total;
  // what a step uploads, in ints from `up`: per slot the lengths of the late layers' rows and of the front layers', tokens of either, the late rows' places
  // among the front rows, the requests' last rows
  size_t start[2], count[2], tokens[2], from, last, up_ints;
};
bool paged_layout(const dmtd_config& c, int wide, int page, PagedLayout& w) {
  if (!page_size_ok(page)) return false;
  const long S = c.max_seq_len, B = c.max_batch;
  w.page = page;
  w.max_pages = (int)((S + page - 1) / page);
  w.n_pages = (int)std::min<long>(B * S / page, INT_MAX);
  w.rows = row_capacity(c, wide);
  if (w.n_pages < 1 || B > kPagedMaxRequests || (long)w.max_pages * page > (1L << 30) || w.rows > (1 << 24)) return false;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
  w.table = take((size_t)B * w.max_pages * 4);
  w.held = take(B * 4);
  w.free_pages = take((size_t)w.n_pages * 4);
  w.n_free = take(4);
  size_t up = 0;
  auto ints = [&](size_t n) { const size_t o = up; up += n; return o; };
  for (int i = 0; i < 2; ++i) { w.start[i] = ints(B); w.count[i] = ints(B); }
  for (int i = 0; i < 2; ++i) w.tokens[i] = ints(w.rows);
  w.from = ints(w.rows);
  w.last = ints(B);
  w.up_ints = up;
  w.up = take(up * 4);
  for (int i = 0; i < 2; ++i) {
    w.cu[i] = take((B + 1) * 4);
    w.pos[i] = take((size_t)w.rows * 4);
    w.slots[i] = take((size_t)w.rows * 8);
  }
  w.status = take((w.kStatus + B) * 4);
  dmtd_paged_cache pc{};
  pc.n_pages = w.n_pages; pc.page_size = page; pc.n_req = (int)B; pc.max_pages = w.max_pages;
  pc.n_q_heads = c.n_q_heads; pc.n_kv_heads = c.n_kv_heads; pc.head_dim = c.head_dim; pc.dtype = c.dtype; pc.max_rows = w.rows;
  const PagedPlan p = paged_plan(&pc, w.rows);
  w.attention_bytes = p.count_bytes + p.few_bytes + p.tall_bytes;
  w.attention = take(w.attention_bytes);
  w.total = off;
  return true;
}

dmtd_page_pool paged_pool(const dmtd_ctx* c, const PagedLayout& w) {
  char* m = c->paged.mem;
  return dmtd_page_pool{w.n_pages, w.page, c->cfg.max_batch, w.max_pages, (int*)(m + w.table), (int*)(m + w.held), (int*)(m + w.free_pages), (int*)(m + w.n_free)};
}

// Pages and places of pass `which` (0: the late layers' rows, 1: the front layers') of so many rows from the uploaded lengths
int paged_tables(dmtd_ctx* c, const PagedLayout& w, int which, int rows) {
  char* m = c->paged.mem;
  const dmtd_page_pool pool = paged_pool(c, w);
  const int* up = (const int*)(m + w.up);
  const int rc = dmtd_page_tables(&pool, up + w.start[which], up + w.count[which], rows, (int*)(m + w.cu[which]), (int*)(m + w.pos[which]), (int64_t*)(m + w.slots[which]),
                                  (int*)(m + w.status) + 2 * which, c->stream);
  if (rc != DMTD_OK) c->err = g_create_error;
  return rc;
}

// The device's word on the tables of a pass: it refuses what does not fit the pool, and the host has checked that the step does
int paged_status(dmtd_ctx* c, const int32_t* status) {
  if (status[0] == 0) return DMTD_OK;
  c->err = "the pool's tables on the device are not those of the steps so far: their memory was written to";
  return DMTD_EHIP;
}

hipError_t paged_layers(dmtd_ctx* c, const PagedLayout& w, int which, Rows& R, int rows, int max_new, int first, int end) {
  PagedPass pass{};
  dmtd_paged_cache& pc = pass.cache;
  char* m = c->paged.mem;
  pc.block_table = (const int*)(m + w.table);
  pc.n_pages = w.n_pages; pc.page_size = w.page; pc.n_req = c->cfg.max_batch; pc.max_pages = w.max_pages;
  pc.n_q_heads = c->cfg.n_q_heads; pc.n_kv_heads = c->cfg.n_kv_heads; pc.head_dim = c->cfg.head_dim; pc.dtype = c->cfg.dtype; pc.max_rows = rows;
  pass.cu = (const int*)(m + w.cu[which]);
  pass.start = (const int*)(m + w.up) + w.start[which];
  pass.pos = (const int*)(m + w.pos[which]);
  pass.slots = (const int64_t*)(m + w.slots[which]);
  pass.max_new = max_new;
  pass.ws = m + w.attention;
  c->batch = 1;                        // the rows of all requests as one sequence's
  c->paged_pass = &pass;
  hipError_t e = hipSuccess;
  for (int l = first; l < end && e == hipSuccess; ++l) e = run_layer(c, l, R, rows, POS_EXPLICIT, 0);
  c->paged_pass = nullptr;
  c->batch = 0;
  return e;
}

// A failure injected from the host (DMTD_TEST_FAIL_STEP at create), midway in a paged call, the way a refused launch would fail it; what was enqueued completes normally
bool paged_injected(dmtd_ctx* c) {
  if (c->test_fail_step < 0 || c->test_fail_step-- > 0) return false;
  c->err = "injected launch failure (DMTD_TEST_FAIL_STEP)";
  return true;
}

// A pass of a step's front layers: per slot where its rows start and their number, the rows' tokens, which of them are new, the most of one slot
struct PagedFront {
  struct Run { int first, n; };
  std::vector<int32_t> lengths, tokens;
  std::vector<Run> kept;
  int max_new = 0;
};

// The host ran out of memory inside a call: what the device has done of it is not known
int paged_no_memory(dmtd_ctx* c) {
  c->paged.failed = true;
  (void)hipStreamSynchronize(c->stream);
  return DMTD_EHIP;
}

}  // namespace

extern "C" {

size_t dmtd_paged_step_bytes(const dmtd_config* cfg, int32_t page_size) {
  std::string why;
  PagedLayout w{};
  if (!valid_config(cfg, why)) return 0;
  return paged_layout(*cfg, kWideRows, page_size, w) ? w.total : 0;
}

int dmtd_paged_begin(dmtd_ctx* c, int32_t page_size, void* memory_dev, size_t memory_bytes) try {
  if (!c) return DMTD_EINVAL;
  const dmtd_config& cf = c->cfg;
  PagedLayout w{};
  if (!paged_layout(cf, c->wide_rows, page_size, w)) { c->err = "page_size must be 16, 32, 64, 128 or 256, and the cache hold a page"; return DMTD_EINVAL; }
  if (cf.dry_run) { c->err = "no device work in a dry run"; return DMTD_ESTATE; }
  if (!memory_dev || !aligned(memory_dev, 256)) { c->err = "memory must be a 256-byte aligned device pointer"; return DMTD_EINVAL; }
  if (c->sched.n_tok != 0 || c->paged.on) { c->err = "paged steps need an empty context; call dmtd_reset first"; return DMTD_ESTATE; }
  if (c->sched.n_early != 0) { c->err = "paged steps are not available in the ExDy variant"; return DMTD_ESTATE; }
  if (memory_bytes < w.total) { c->err = "memory too small"; return DMTD_ECAPACITY; }
  // Empty tables, every page free, the attention's counters 0
  std::vector<int32_t> table((size_t)cf.max_batch * w.max_pages, -1), zeros(cf.max_batch, 0), free_pages(w.n_pages);
  for (int i = 0; i < w.n_pages; ++i) free_pages[i] = w.n_pages - 1 - i;
  char* m = (char*)memory_dev;
  HIP_TRY(c, hipMemcpyAsync(m + w.table, table.data(), table.size() * 4, hipMemcpyHostToDevice, c->stream));
  HIP_TRY(c, hipMemcpyAsync(m + w.held, zeros.data(), zeros.size() * 4, hipMemcpyHostToDevice, c->stream));
  HIP_TRY(c, hipMemcpyAsync(m + w.free_pages, free_pages.data(), free_pages.size() * 4, hipMemcpyHostToDevice, c->stream));
  HIP_TRY(c, hipMemcpyAsync(m + w.n_free, &w.n_pages, 4, hipMemcpyHostToDevice, c->stream));
  HIP_TRY(c, hipMemsetAsync(m + w.attention, 0, w.attention_bytes, c->stream));
  HIP_TRY(c, hipStreamSynchronize(c->stream));
  c->paged = PagedState{};
  c->paged.on = true;
  c->paged.page = page_size;
  c->paged.mem = m;
  c->paged.free_pages = w.n_pages;
  c->paged.seqs.resize(cf.max_batch);
  return DMTD_OK;
} catch (const std::bad_alloc&) { return paged_no_memory(c); }

int dmtd_paged_step(dmtd_ctx* c, int32_t n, const int32_t* slots, const int32_t* counts, const int32_t* tokens, const uint8_t* full, int32_t n_late,
                    int32_t* next_tokens) try {
  if (!c) return DMTD_EINVAL;
  const dmtd_config& cf = c->cfg;
  if (!c->paged.on) { c->err = "dmtd_paged_step before dmtd_paged_begin"; return DMTD_ESTATE; }
  if (c->paged.failed) { c->err = "a paged step failed midway; call dmtd_reset"; return DMTD_ESTATE; }
  if (c->sampling) { c->err = "paged steps select greedily"; return DMTD_ESTATE; }
  if (!slots || !counts || !tokens || !full) { c->err = "null pointer"; return DMTD_EINVAL; }
  if (n < 1 || n > cf.max_batch) { c->err = "number of requests outside [1, max_batch]"; return DMTD_EINVAL; }
  if (n_late < 1 || n_late > cf.n_layers) { c->err = "n_late must be in [1, n_layers]"; return DMTD_EINVAL; }
  PagedLayout w{};
  paged_layout(cf, c->wide_rows, c->paged.page, w);
  std::vector<PagedState::Seq>& seqs = c->paged.seqs;
  std::vector<int> request(cf.max_batch, -1);          // of a slot
  std::vector<size_t> first_token(n);
  size_t n_tokens = 0;
  int late_rows_n = 0, take = 0;
  for (int j = 0; j < n; ++j) {
    if (slots[j] < 0 || slots[j] >= cf.max_batch) { c->err = "slot outside [0, max_batch)"; return DMTD_EINVAL; }
    if (request[slots[j]] >= 0) { c->err = "a slot is named twice"; return DMTD_EINVAL; }
    if (counts[j] < 1) { c->err = "a request brings at least one token"; return DMTD_EINVAL; }
    request[slots[j]] = j;
    const PagedState::Seq& q = seqs[slots[j]];
    if (counts[j] > cf.max_seq_len - q.n_tok) { c->err = "a request would exceed max_seq_len"; return DMTD_ECAPACITY; }
    if (counts[j] > w.rows - late_rows_n) { c->err = "more rows than a pass carries"; return DMTD_ECAPACITY; }
    late_rows_n += counts[j];
    first_token[j] = n_tokens;
    for (int i = 0; i < counts[j]; ++i, ++n_tokens)
      if (tokens[n_tokens] < 0 || tokens[n_tokens] >= cf.vocab) { c->err = "token id outside the vocabulary"; return DMTD_EINVAL; }
    take += (q.n_tok + counts[j] + w.page - 1) / w.page - (q.n_tok + w.page - 1) / w.page;
  }
  if (take > c->paged.free_pages) { c->err = "the pool lacks pages"; return DMTD_ECAPACITY; }
  if (c->paged.n_late != 0 && c->paged.n_late != n_late)
    for (const PagedState::Seq& q : seqs)
      if (!q.pending.empty()) { c->err = "n_late changed while tokens await refill"; return DMTD_ESTATE; }
  // The rows in the order of the slots.  The front layers' rows may take several passes: a request that the last pass does not hold whole begins one, and fills several where no pass holds it; behind its
  // last part others follow.  Lengths say what pages a request holds, so the first of several parts gives back those of the later ones; nobody else takes or gives any until these, pass by
  // pass, have taken them off the stack again, in their order.
  const int F = cf.n_layers - n_late;
  std::vector<int32_t> up(w.up_ints, 0);
  std::vector<PagedFront> fronts;
  auto new_front = [&]() {
    fronts.emplace_back();
    PagedFront& f = fronts.back();
    f.lengths.resize(w.count[1] + cf.max_batch - w.start[1], 0);
    for (int s = 0; s < cf.max_batch; ++s) f.lengths[s] = seqs[s].n_tok + (request[s] >= 0 ? counts[request[s]] : 0);       // (no rows: it keeps its pages)
  };
  std::vector<int32_t> from;           // where several passes leave their results at the new tokens: behind one another
  int late_at = 0, kept_at = 0, max_late = 0;
  bool same = true, any_full = false;                    // the front layers' rows are the late layers'
  for (int s = 0; s < cf.max_batch; ++s) {
    const PagedState::Seq& q = seqs[s];
    const int j = request[s], count = j >= 0 ? counts[j] : 0, rows = j >= 0 && full[j] ? (int)q.pending.size() + count : 0;
    up[w.start[0] + s] = q.n_tok;
    up[w.count[0] + s] = count;
    same = same && rows == count;
    any_full = any_full || rows;
    if (F > 0)
      for (int at = 0; at < rows;) {
        if (fronts.empty() || (int)fronts.back().tokens.size() + (at ? 0 : std::min(rows, w.rows)) > w.rows) new_front();
        PagedFront& f = fronts.back();
        const int n_rows = std::min(rows - at, w.rows), pending = (int)q.pending.size();
        f.lengths[s] = q.n_front + at;
        f.lengths[w.count[1] - w.start[1] + s] = n_rows;
        f.max_new = std::max(f.max_new, n_rows);
        const int fresh = std::max(at, pending);
        if (at + n_rows > fresh) f.kept.push_back({(int)f.tokens.size() + fresh - at, at + n_rows - fresh});
        for (int i = at; i < at + n_rows; ++i) f.tokens.push_back(i < pending ? q.pending[i] : tokens[first_token[j] + i - pending]);
        at += n_rows;
        if (at < rows) new_front();
      }
    const int new_at = rows && F > 0 ? (int)fronts.back().tokens.size() - count : 0;      // in one pass: all rows are kept
    for (int i = 0; i < count; ++i) {
      from.push_back(rows ? kept_at++ : -1);
      up[w.from + late_at] = rows ? new_at + i : -1;
      up[w.tokens[0] + late_at++] = tokens[first_token[j] + i];
    }
    if (j >= 0) up[w.last + j] = late_at - 1;
    max_late = std::max(max_late, count);
  }
  if (fronts.size() > 1) {
    std::copy(from.begin(), from.end(), up.begin() + w.from);
  } else if (!fronts.empty()) {
    std::copy(fronts[0].lengths.begin(), fronts[0].lengths.end(), up.begin() + w.start[1]);
    std::copy(fronts[0].tokens.begin(), fronts[0].tokens.end(), up.begin() + w.tokens[1]);
  }
  char* m = c->paged.mem;
  const int* dev = (const int*)(m + w.up);
  const bool add = cf.full_pos_add_embed != 0;
  std::vector<int32_t> next(w.kStatus + n);
  const bool front_tables = !fronts.empty() && !same;
  auto run = [&]() -> int {
    HIP_TRY(c, hipMemcpyAsync(m + w.up, up.data(), up.size() * 4, hipMemcpyHostToDevice, c->stream));
    int rc = paged_tables(c, w, 0, late_rows_n);
    if (rc != DMTD_OK) return rc;
    Rows R = front_rows(c), last = late_rows(c);
    float* kept = (float*)(c->ws + c->o.enc_tmp);        // the front layers' results at the new tokens
    size_t n_kept = 0;
    for (const PagedFront& f : fronts) {
      const int rows = (int)f.tokens.size();
      if (fronts.size() > 1) {
        HIP_TRY(c, hipMemcpyAsync(m + w.up + w.start[1] * 4, f.lengths.data(), f.lengths.size() * 4, hipMemcpyHostToDevice, c->stream));
        HIP_TRY(c, hipMemcpyAsync(m + w.up + w.tokens[1] * 4, f.tokens.data(), f.tokens.size() * 4, hipMemcpyHostToDevice, c->stream));
      }
      if (front_tables && (rc = paged_tables(c, w, 1, rows)) != DMTD_OK) return rc;
      HIP_TRY(c, paged_rows(c, rows, nullptr, nullptr, dev + w.tokens[1], false, R, 0));
      HIP_TRY(c, paged_layers(c, w, same ? 0 : 1, R, rows, f.max_new, 0, F));
      if (fronts.size() == 1) {
        if (!same || add) HIP_TRY(c, hipMemcpyAsync(kept, R.h, (size_t)rows * cf.hidden * 4, hipMemcpyDeviceToDevice, c->stream));
        continue;
      }
      for (const auto& k : f.kept) {
        HIP_TRY(c, hipMemcpyAsync(kept + n_kept * cf.hidden, R.h + (size_t)k.first * cf.hidden, (size_t)k.n * cf.hidden * 4, hipMemcpyDeviceToDevice, c->stream));
        n_kept += k.n;
      }
      int32_t status[2] = {-1, -1};                      // before the next pass's
      HIP_TRY(c, hipMemcpyAsync(status, (int*)(m + w.status) + 2, sizeof(status), hipMemcpyDeviceToHost, c->stream));
      HIP_TRY(c, hipStreamSynchronize(c->stream));
      if ((rc = paged_status(c, status)) != DMTD_OK) return rc;
    }
    if (!fronts.empty()) {
      if (!same || add) HIP_TRY(c, paged_rows(c, late_rows_n, kept, dev + w.from, dev + w.tokens[0], add, R, F));
    } else {
      HIP_TRY(c, paged_rows(c, late_rows_n, nullptr, nullptr, dev + w.tokens[0], false, R, F));
      // no front layers: the literal reading adds the embedding once more at full positions
      if (add && any_full) {
        HIP_TRY(c, hipMemcpyAsync(kept, R.h, (size_t)late_rows_n * cf.hidden * 4, hipMemcpyDeviceToDevice, c->stream));
        std::vector<int32_t> twice(late_rows_n);
        for (int i = 0; i < late_rows_n; ++i) twice[i] = up[w.from + i] >= 0 ? i : -1;
        HIP_TRY(c, hipMemcpyAsync(m + w.up + w.from * 4, twice.data(), twice.size() * 4, hipMemcpyHostToDevice, c->stream));
        HIP_TRY(c, hipStreamSynchronize(c->stream));
        HIP_TRY(c, paged_rows(c, late_rows_n, kept, dev + w.from, dev + w.tokens[0], true, R, F));
      }
    }
    HIP_TRY(c, paged_layers(c, w, 0, R, late_rows_n, max_late, F, cf.n_layers));
    HIP_TRY(c, paged_rows(c, n, R.h, dev + w.last, nullptr, false, last, cf.n_layers));
    HIP_TRY(c, head_logits(c, last, n, (float*)(c->ws + c->o.logits), c->amax, cf.max_batch));
    if (paged_injected(c)) return DMTD_EHIP;
    hipLaunchKernelGGL(paged_pick_kernel, dim3(n), dim3(64), 0, c->stream, c->amax, AMAX_CELLS, cf.max_batch, (int*)(m + w.status) + w.kStatus);
    HIP_TRY(c, hipGetLastError());
    HIP_TRY(c, hipMemcpyAsync(next.data(), m + w.status, next.size() * 4, hipMemcpyDeviceToHost, c->stream));
    HIP_TRY(c, hipStreamSynchronize(c->stream));
    if ((rc = paged_status(c, next.data())) == DMTD_OK && front_tables) rc = paged_status(c, next.data() + 2);
    return rc;
  };
  const int rc = run();
  if (rc != DMTD_OK) { c->paged.failed = true; (void)hipStreamSynchronize(c->stream); return rc; }
  for (int s = 0; s < cf.max_batch; ++s) {
    const int j = request[s];
    if (j < 0) continue;
    PagedState::Seq& q = seqs[s];
    q.n_tok += counts[j];
    if (full[j]) {
      q.n_front = q.n_tok;
      q.pending.clear();
    } else {
      q.pending.insert(q.pending.end(), tokens + first_token[j], tokens + first_token[j] + counts[j]);
    }
  }
  c->paged.free_pages -= take;
  c->paged.n_late = n_late;
  c->paged.last_n = n;
  if (next_tokens) std::memcpy(next_tokens, next.data() + w.kStatus, (size_t)n * 4);
  return DMTD_OK;
} catch (const std::bad_alloc&) { return paged_no_memory(c); }

int dmtd_paged_release(dmtd_ctx* c, int32_t slot) try {
  if (!c) return DMTD_EINVAL;
  if (!c->paged.on) { c->err = "dmtd_paged_release before dmtd_paged_begin"; return DMTD_ESTATE; }
  if (c->paged.failed) { c->err = "a paged step failed midway; call dmtd_reset"; return DMTD_ESTATE; }
  if (slot < 0 || slot >= c->cfg.max_batch) { c->err = "slot outside [0, max_batch)"; return DMTD_EINVAL; }
  PagedLayout w{};
  paged_layout(c->cfg, c->wide_rows, c->paged.page, w);
  PagedState::Seq& q = c->paged.seqs[slot];
  std::vector<int32_t> up(2 * (size_t)c->cfg.max_batch, 0);          // lengths, no rows
  for (int s = 0; s < c->cfg.max_batch; ++s) up[s] = s == slot ? 0 : c->paged.seqs[s].n_tok;
  auto run = [&]() -> int {
    HIP_TRY(c, hipMemcpyAsync(c->paged.mem + w.up + w.start[0] * 4, up.data(), up.size() * 4, hipMemcpyHostToDevice, c->stream));
    const int rc = paged_tables(c, w, 0, 1);
    if (rc != DMTD_OK) return rc;
    if (paged_injected(c)) return DMTD_EHIP;
    int32_t status[2] = {-1, -1};
    HIP_TRY(c, hipMemcpyAsync(status, c->paged.mem + w.status, sizeof(status), hipMemcpyDeviceToHost, c->stream));
    HIP_TRY(c, hipStreamSynchronize(c->stream));
    return paged_status(c, status);
  };
  const int rc = run();
  if (rc != DMTD_OK) { c->paged.failed = true; (void)hipStreamSynchronize(c->stream); return rc; }
  c->paged.free_pages += (q.n_tok + w.page - 1) / w.page;
  q = PagedState::Seq{};
  return DMTD_OK;
} catch (const std::bad_alloc&) { return paged_no_memory(c); }

int dmtd_paged_get_state(const dmtd_ctx* c, int32_t slot, int32_t* n_tok, int32_t* n_front, int32_t* free_pages) {
  if (!c || !c->paged.on || slot < 0 || slot >= c->cfg.max_batch) return DMTD_EINVAL;
  if (n_tok) *n_tok = c->paged.seqs[slot].n_tok;
  if (n_front) *n_front = c->paged.seqs[slot].n_front;
  if (free_pages) *free_pages = c->paged.free_pages;
  return DMTD_OK;
}

}  // extern "C"
