// Attention of a step's new tokens over the paged cache of their requests (paged.hpp).  The new tokens' own keys and values are in the cache
// already (paged_append_kernel); row t of request i, at position start[i] + t, sees the request's keys 0 .. start[i] + t.
#pragma once
#include "paged.hpp"

namespace dmtd {

// Rows of a request as the kernels read them: none where the lengths do not fit the buffers or the tables
struct PagedReq { int first, n, start; };
__device__ __forceinline__ PagedReq paged_req(const PagedView& pv, const int* cu, const int* start, int max_new, int i) {
  PagedReq q{cu[i], cu[i + 1] - cu[i], start[i]};
  if (q.first < 0 || q.n < 0 || q.n > max_new || q.first > pv.max_rows - q.n || q.start < 0 || q.start > pv.limit - q.n) q.n = 0;
  return q;
}

// One block per (row, query head); its 4 waves take 64 keys each in turn, a lane scores one key and then carries HD / 64 dims of the output.
template <typename CT, int HD>
__global__ void __launch_bounds__(256) paged_attention_rows_kernel(const float* __restrict__ qkv, long ld, const int* __restrict__ start, const int* __restrict__ cu,
                                                                   const CT* __restrict__ q_gain, const float2* __restrict__ rope_tab, float eps, int max_new,
                                                                   CT* __restrict__ out, long ldo, PagedView pv) {
  constexpr int half = HD / 2, DPL = HD / 64;
  __shared__ __attribute__((aligned(16))) float q_s[HD];
  __shared__ float o_s[4][HD], m_s[4], l_s[4];
  const int t = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (t >= cu[pv.n_req] || t < cu[0]) return;
  const int i = last_at_most(cu, pv.n_req, t);
  const PagedReq rq = paged_req(pv, cu, start, max_new, i);
  if (t >= rq.first + rq.n) return;
  const int pos = rq.start + t - rq.first;
  const int g = head / (pv.nh / pv.nkv);
  if (wave == 0) {
    const float* src = qkv + (size_t)t * ld + (size_t)head * HD;
    const bool act = lane < half;
    float a = act ? src[lane] : 0.f, b = act ? src[lane + half] : 0.f;
    const float rs = q_gain ? rsqrtf(wave_sum(a * a + b * b) / (float)HD + eps) : 1.f;
    if (act) {
      if (q_gain) { a *= rs * Elem<CT>::to_f32(q_gain[lane]); b *= rs * Elem<CT>::to_f32(q_gain[lane + half]); }
      const float2 cs = rope_tab ? rope_tab[(size_t)pos * half + lane] : make_float2(1.f, 0.f);
      const float scale = rsqrtf((float)HD);
      q_s[lane] = (a * cs.x - b * cs.y) * scale;
      q_s[lane + half] = (b * cs.x + a * cs.y) * scale;
    }
  }
  __syncthreads();
  const int* table = pv.table + (size_t)i * pv.max_pages;
  auto at = [&](int key, int page) { return (size_t)page * pv.page_stride + (((size_t)g << pv.page_shift) + (key & ((1 << pv.page_shift) - 1))) * HD; };
  float m = -INFINITY, l = 0.f, acc[DPL];
#pragma unroll
  for (int e = 0; e < DPL; ++e) acc[e] = 0.f;
  for (int base = 64 * wave; base <= pos; base += 256) {
    const int key = base + lane;
    const int page = key <= pos ? table[key >> pv.page_shift] : -1;
    const bool seen = page >= 0 && page < pv.n_pages;
    float s = -INFINITY;
    if (seen) {
      const CT* kp = (const CT*)pv.k + at(key, page);
      s = 0.f;
      for (int d = 0; d < HD; d += 8) {
        float w[8];
        Elem<CT>::load8(kp + d, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += w[e] * q_s[d + e];
      }
    }
    const float m_new = fmaxf(m, wave_max(s)), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float p = seen ? __expf(s - m_use) : 0.f, f = __expf(m - m_use);
    m = m_new;
    l = l * f + wave_sum(p);
#pragma unroll
    for (int e = 0; e < DPL; ++e) acc[e] *= f;
    for (int kk = 0; kk < 64 && base + kk <= pos; ++kk) {
      const int pg = __shfl(page, kk, 64);
      const float pk = __shfl(p, kk, 64);
      if (pg < 0 || pg >= pv.n_pages) continue;
      const CT* vp = (const CT*)pv.v + at(base + kk, pg) + DPL * lane;
#pragma unroll
      for (int e = 0; e < DPL; ++e) acc[e] += pk * Elem<CT>::to_f32(vp[e]);
    }
  }
  if (lane == 0) { m_s[wave] = m; l_s[wave] = l; }
#pragma unroll
  for (int e = 0; e < DPL; ++e) o_s[wave][DPL * lane + e] = acc[e];
  __syncthreads();
  if (threadIdx.x < HD) {
    const int d = threadIdx.x;
    const float mm = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3])), mu = mm == -INFINITY ? 0.f : mm;
    float o = 0.f, ll = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __expf(m_s[w] - mu);
      o += f * o_s[w][d];
      ll += f * l_s[w];
    }
    out[(size_t)t * ldo + (size_t)head * HD + d] = Elem<CT>::from_f32(ll == 0.f ? 0.f : o / ll);
  }
}

}  // namespace dmtd
