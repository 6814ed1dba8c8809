// Attention of new tokens over a paged cache (adept_paged_attend).
//
// One wave per (entry, head) walks the entry's keys one after another: lane l
// holds the dims l, l + 64, ... of q and of the running output, a score is a
// sum over the wave, and the softmax keeps a running maximum and sum, so the
// keys are read once.  A key that is not seen is skipped, whatever it holds.
#include "paged.h"

namespace adept {
namespace {

// value d of the (slot, head) row `row` of a cache, row = slot * Hkv + head
template <typename TC>
__device__ __forceinline__ float cache_value(const void* c, const uint8_t* scale, int64_t row,
                                             int hd, int d) {
  if constexpr (sizeof(TC) == 1) {
    const uint32_t w = ((const uint8_t*)c)[row * hd + d];
    return fp8x2_to_f32x2<false>(w, scale_of(scale[row])).x;
  } else {
    return ld((const TC*)c + row * hd + d);
  }
}

template <typename T, typename TC>
__global__ __launch_bounds__(256) void paged_attend_wave_kernel(int H, int hd, float scale_log2,
                                                                const T* __restrict__ q, Entries e,
                                                                PagedView c, T* __restrict__ out) {
  const int k = blockIdx.x, h = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (k >= min(*e.n_active, e.max_active) || h >= H) return;
  int b;
  const int n = entry_limit(e, c, e.rows[k], &b);
  const int32_t* pages = c.table + (int64_t)b * c.max_pages;
  const int hk = h / (H / c.n_kv_heads);
  const int64_t at = ((int64_t)k * H + h) * hd;
  float qv[4], o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = lane + 64 * i;
    qv[i] = d < hd ? ld(q + at + d) * scale_log2 : 0.0f;
    o[i] = 0.0f;
  }
  float m = -INFINITY, l = 0.0f;
  for (int t = 0; t < n; ++t) {
    const int s = c.slot(pages, t);
    if (s < 0) continue;
    const int64_t row = (int64_t)s * c.n_kv_heads + hk;
    float x = 0.0f, v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      v[i] = 0.0f;
      if (d >= hd) continue;
      x = fmaf(qv[i], cache_value<TC>(c.k, c.k_scale, row, hd, d), x);
      v[i] = cache_value<TC>(c.v, c.v_scale, row, hd, d);
    }
    x = wave_sum_f32(x);
    if (x == -INFINITY) continue;      // no weight
    const float mn = fmaxf(m, x);
    const float a = exp2f(m - mn), p = exp2f(x - mn);
    m = mn;
    l = fmaf(l, a, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = fmaf(p, v[i], o[i] * a);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // no key: zeros
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 64 * i < hd) st(out + at + lane + 64 * i, o[i] * inv);
}

}  // namespace
}  // namespace adept

using namespace adept;

extern "C" size_t adept_paged_attend_workspace_bytes(const adept_paged_kv* kv, int n_heads,
                                                     int max_active, int n_seq, int max_pages) {
  (void)kv; (void)n_heads; (void)max_active; (void)n_seq; (void)max_pages;
  return 256;
}

extern "C" adept_status adept_paged_attend(adept_dtype dt, const adept_paged_kv* kv, int n_heads,
                                           float scale, int causal, const void* q,
                                           const int32_t* rows, const int32_t* n_active,
                                           int max_active, const int32_t* pos, const int32_t* seq,
                                           int n_seq, const int32_t* page_table, int max_pages,
                                           const int32_t* key_len, const uint8_t* key_live,
                                           void* out, void* workspace, size_t workspace_bytes,
                                           void* stream) {
  ADEPT_TRY(paged_check("paged_attend", dt, kv));
  const int hd = kv->head_dim;
  ADEPT_REQUIRE(n_heads > 0 && n_heads <= 4096 && n_heads % kv->n_kv_heads == 0,
                "paged_attend: %d heads are no multiple of %d", n_heads, kv->n_kv_heads);
  ADEPT_REQUIRE(max_active >= 0 && max_active <= kMaxEntries && n_seq > 0 && max_pages > 0 &&
                    (int64_t)max_pages * kv->page_size <= INT_MAX,
                "paged_attend: bad sizes");
  if (max_active == 0) return ADEPT_OK;
  ADEPT_REQUIRE(q && rows && n_active && pos && seq && page_table && out,
                "paged_attend: NULL tensor");
  ADEPT_REQUIRE(causal == 1 || (causal == 0 && key_len),
                "paged_attend: bidirectional attention needs key_len");
  ADEPT_REQUIRE(aligned16(q) && aligned16(out), "paged_attend: q and out must be 16-byte aligned");
  ADEPT_REQUIRE(scale > 0.0f && scale < INFINITY, "paged_attend: scale must be positive");
  const size_t need = adept_paged_attend_workspace_bytes(kv, n_heads, max_active, n_seq, max_pages);
  if (!workspace || !aligned16(workspace) || workspace_bytes < need) {
    set_error("paged_attend: workspace of %zu bytes needed, 16-byte aligned", need);
    return ADEPT_E_WORKSPACE;
  }
  int shift = 0;
  while ((1 << shift) < kv->page_size) ++shift;
  const PagedView c{kv->k, kv->v, kv->k_scale, kv->v_scale, page_table, key_live, max_pages,
                    kv->n_pages, shift, kv->n_kv_heads, n_seq};
  const Entries e{rows, n_active, pos, seq, key_len, max_active, causal};
  const float sl = scale * 1.4426950408889634f;   // scores in the exp2 domain
  hipStream_t s = as_stream(stream);
  const dim3 grid(max_active, ceil_div(n_heads, 4));
#define ADEPT_WAVE(T, TC)                                                                       \
  ADEPT_LAUNCH((paged_attend_wave_kernel<T, TC>), grid, dim3(256), 0, s, n_heads, hd, sl,       \
               (const T*)q, e, c, (T*)out)
  const bool fp8 = kv->dtype == ADEPT_KV_FP8;
  if (dt == ADEPT_F32) {
    if (fp8) ADEPT_WAVE(float, uint8_t); else ADEPT_WAVE(float, float);
  } else {
    if (fp8) ADEPT_WAVE(bf16, uint8_t); else ADEPT_WAVE(bf16, bf16);
  }
#undef ADEPT_WAVE
  return launch_status("paged_attend");
}
