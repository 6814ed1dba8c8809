// Rows written into a paged cache and read back (adept_paged_store,
// adept_paged_load): copied, or quantised to e4m3 with one power-of-two scale
// per (slot, head) row.
//
// A row of hd values belongs to hd/8 neighbouring lanes, eight values each, K
// and V in the same thread.  Quantising needs the row's largest magnitude
// before anything is written: lane shuffles over the row's lanes, with the
// values kept in registers, so the row crosses HBM once each way.
//
// Bound by HBM.  What the caller hands in and what it gets back passes through
// once, by non-temporal loads and stores; the cache's own lines do not, they are
// soon read again: 8192 rows of 32x128 bf16 stored in 8 bits and read back 67 us
// (5.0 TB/s, a large copy's rate; 84 with all accesses ordinary, 79 with all
// non-temporal), 20011 rows read back 86 us (5.7 TB/s; 98).
#include "paged.h"

namespace adept {

adept_status paged_check(const char* what, adept_dtype dt, const adept_paged_kv* kv) {
  ADEPT_REQUIRE(dt == ADEPT_F32 || dt == ADEPT_BF16, "%s: bad dtype", what);
  ADEPT_REQUIRE(kv != nullptr, "%s: NULL cache", what);
  ADEPT_REQUIRE(kv->dtype == ADEPT_KV_FP8 || kv->dtype == (dt == ADEPT_F32 ? ADEPT_KV_F32 : ADEPT_KV_BF16),
                "%s: cache type %d does not go with dtype %d", what, kv->dtype, (int)dt);
  ADEPT_REQUIRE(kv->n_kv_heads > 0 && kv->n_kv_heads <= 4096, "%s: bad n_kv_heads %d", what,
                kv->n_kv_heads);
  const int hd = kv->head_dim, ps = kv->page_size;
  ADEPT_REQUIRE(hd >= 16 && hd <= 256 && (hd & (hd - 1)) == 0,
                "%s: head_dim %d must be a power of two from 16 to 256", what, hd);
  ADEPT_REQUIRE(ps >= 1 && ps <= 1024 && (ps & (ps - 1)) == 0,
                "%s: page_size %d must be a power of two from 1 to 1024", what, ps);
  ADEPT_REQUIRE(kv->n_pages > 0 && paged_slots(*kv) <= kMaxTokens, "%s: bad n_pages %d", what,
                kv->n_pages);
  ADEPT_REQUIRE(kv->k && kv->v && aligned16(kv->k) && aligned16(kv->v),
                "%s: K and V must be 16-byte aligned", what);
  ADEPT_REQUIRE(kv->dtype != ADEPT_KV_FP8 || (kv->k_scale && kv->v_scale),
                "%s: an FP8 cache needs its scales", what);
  return ADEPT_OK;
}

namespace {

constexpr int kThreads = 256;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4_t load_once(const void* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
}
__device__ __forceinline__ void store_once(void* p, u32x4_t x) {
  __builtin_nontemporal_store(x, reinterpret_cast<u32x4_t*>(p));
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    const u32x4_t w = load_once(p + e);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[e + i] = __uint_as_float(w[i]);
  }
}
__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const u32x4_t w = load_once(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}

// Scale byte of a row whose largest finite magnitude has the bits `top`:
// with top = m 2^x, 1 <= m < 2, the least E with top <= 448 2^E = 1.75 2^(E+8)
// is x - 8 where m <= 1.75, else x - 7.
__device__ __forceinline__ int scale_byte(uint32_t top) {
  const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kScaleMin), kScaleMax);
}

// Eight values of a row that lanes share (lpr of them, neighbours): the codes
// and the row's scale byte.
__device__ __forceinline__ uint2 quantise8(const float (&x)[8], int lpr, int* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t a = __float_as_uint(x[e]) & 0x7fffffffu;
    top = max(top, a < 0x7f800000u ? a : 0u);   // magnitudes order as their bits
  }
  for (int o = lpr >> 1; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  *byte = scale_byte(top);
  const float inv = __uint_as_float((uint32_t)(254 - *byte) << 23);
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool fine = (__float_as_uint(x[e]) & 0x7fffffffu) < 0x7f800000u;
    y[e] = fine ? fminf(fmaxf(x[e] * inv, -448.0f), 448.0f) : __uint_as_float(0x7fc00000u);
  }
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

template <typename T, bool FP8>
__global__ __launch_bounds__(kThreads) void paged_store_kernel(
    int heads, int hd, const T* __restrict__ k, int64_t k_stride, const T* __restrict__ v,
    int64_t v_stride, const int32_t* __restrict__ rows, const int32_t* __restrict__ n_rows,
    int max_rows, const int32_t* __restrict__ slot, int n_slots, void* kc, void* vc,
    uint8_t* __restrict__ ks, uint8_t* __restrict__ vs) {
  const int i = blockIdx.x;
  const int n = n_rows ? min(*n_rows, max_rows) : max_rows;
  if (i >= n) return;
  const int j = rows ? rows[i] : i;
  const int s = slot[j];
  if ((unsigned)s >= (unsigned)n_slots) return;
  const int lpr = hd >> 3;                        // lanes per head row
  const int c = blockIdx.y * kThreads + threadIdx.x;   // eight values of the token's row
  if (c >= heads * lpr) return;                   // whole head rows: lpr divides the block
  const int64_t at = (int64_t)s * heads * hd + c * 8;
  const T* kp = k + j * k_stride + c * 8;
  const T* vp = v + j * v_stride + c * 8;
  if constexpr (FP8) {
    float x[8], y[8];
    load8(kp, x);
    load8(vp, y);
    int kb, vb;
    const uint2 kq = quantise8(x, lpr, &kb), vq = quantise8(y, lpr, &vb);
    *reinterpret_cast<uint2*>((uint8_t*)kc + at) = kq;
    *reinterpret_cast<uint2*>((uint8_t*)vc + at) = vq;
    if (c % lpr == 0) {
      ks[(int64_t)s * heads + c / lpr] = (uint8_t)kb;
      vs[(int64_t)s * heads + c / lpr] = (uint8_t)vb;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += 16 / sizeof(T)) {
      const u32x4_t a = load_once(kp + e), b = load_once(vp + e);
      *reinterpret_cast<u32x4_t*>((T*)kc + at + e) = a;
      *reinterpret_cast<u32x4_t*>((T*)vc + at + e) = b;
    }
  }
}

__device__ __forceinline__ void expand8(uint2 w, float scale, bf16* out) {
  store_once(out, u32x4_t{fp8x2_to_bf16x2<false>(w.x, scale), fp8x2_to_bf16x2<true>(w.x, scale),
                          fp8x2_to_bf16x2<false>(w.y, scale), fp8x2_to_bf16x2<true>(w.y, scale)});
}
__device__ __forceinline__ void expand8(uint2 w, float scale, float* out) {
  const float2 a = fp8x2_to_f32x2<false>(w.x, scale), b = fp8x2_to_f32x2<true>(w.x, scale);
  const float2 c = fp8x2_to_f32x2<false>(w.y, scale), d = fp8x2_to_f32x2<true>(w.y, scale);
  store_once(out, u32x4_t{__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x),
                          __float_as_uint(b.y)});
  store_once(out + 4, u32x4_t{__float_as_uint(c.x), __float_as_uint(c.y), __float_as_uint(d.x),
                              __float_as_uint(d.y)});
}

template <typename T, bool FP8>
__global__ __launch_bounds__(kThreads) void paged_load_kernel(
    int heads, int hd, const void* __restrict__ kc, const void* __restrict__ vc,
    const uint8_t* __restrict__ ks, const uint8_t* __restrict__ vs,
    const int32_t* __restrict__ slot, const int32_t* __restrict__ n_rows, int max_rows, int n_slots,
    T* __restrict__ k, int64_t k_stride, T* __restrict__ v, int64_t v_stride) {
  const int i = blockIdx.x;
  const int n = n_rows ? min(*n_rows, max_rows) : max_rows;
  if (i >= n) return;
  const int lpr = hd >> 3;
  const int c = blockIdx.y * kThreads + threadIdx.x;
  if (c >= heads * lpr) return;
  const int s = slot[i];
  T* ko = k + i * k_stride + c * 8;
  T* vo = v + i * v_stride + c * 8;
  const bool there = (unsigned)s < (unsigned)n_slots;
  const int64_t at = (int64_t)s * heads * hd + c * 8;
  if constexpr (FP8) {
    uint2 a = make_uint2(0, 0), b = a;
    float sa = 1.0f, sb = 1.0f;
    if (there) {
      a = *reinterpret_cast<const uint2*>((const uint8_t*)kc + at);
      b = *reinterpret_cast<const uint2*>((const uint8_t*)vc + at);
      sa = scale_of(ks[(int64_t)s * heads + c / lpr]);
      sb = scale_of(vs[(int64_t)s * heads + c / lpr]);
    }
    expand8(a, sa, ko);
    expand8(b, sb, vo);
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += 16 / sizeof(T)) {
      u32x4_t a = {0, 0, 0, 0}, b = a;
      if (there) {
        a = *reinterpret_cast<const u32x4_t*>((const T*)kc + at + e);
        b = *reinterpret_cast<const u32x4_t*>((const T*)vc + at + e);
      }
      store_once(ko + e, a);
      store_once(vo + e, b);
    }
  }
}

adept_status check_rows(const char* what, adept_dtype dt, const adept_paged_kv* kv, const void* k,
                        int64_t k_stride, const void* v, int64_t v_stride, int max_rows,
                        const int32_t* slot) {
  ADEPT_TRY(paged_check(what, dt, kv));
  ADEPT_REQUIRE(max_rows >= 0 && max_rows <= kMaxEntries, "%s: bad max_rows %d", what, max_rows);
  if (max_rows == 0) return ADEPT_OK;
  ADEPT_REQUIRE(k && v && slot, "%s: NULL tensor", what);
  const int64_t width = (int64_t)kv->n_kv_heads * kv->head_dim;
  const int per16 = dt == ADEPT_F32 ? 4 : 8;
  ADEPT_REQUIRE(aligned16(k) && aligned16(v), "%s: rows must be 16-byte aligned", what);
  ADEPT_REQUIRE(k_stride >= width && v_stride >= width && k_stride % per16 == 0 &&
                    v_stride % per16 == 0,
                "%s: row strides must be multiples of 16 bytes and at least %lld elements", what,
                (long long)width);
  return ADEPT_OK;
}

dim3 row_grid(const adept_paged_kv& kv, int max_rows) {
  return dim3(max_rows, ceil_div((long)kv.n_kv_heads * (kv.head_dim / 8), kThreads));
}

}  // namespace
}  // namespace adept

using namespace adept;

extern "C" adept_status adept_paged_store(adept_dtype dt, const adept_paged_kv* kv, const void* k,
                                          int64_t k_stride, const void* v, int64_t v_stride,
                                          const int32_t* rows, const int32_t* n_rows, int max_rows,
                                          const int32_t* slot, void* stream) {
  ADEPT_TRY(check_rows("paged_store", dt, kv, k, k_stride, v, v_stride, max_rows, slot));
  if (max_rows == 0) return ADEPT_OK;
  const dim3 grid = row_grid(*kv, max_rows);
  const int H = kv->n_kv_heads, hd = kv->head_dim, ns = (int)paged_slots(*kv);
  hipStream_t s = as_stream(stream);
#define ADEPT_STORE(T, FP8)                                                                   \
  ADEPT_LAUNCH((paged_store_kernel<T, FP8>), grid, dim3(kThreads), 0, s, H, hd, (const T*)k,  \
               k_stride, (const T*)v, v_stride, rows, n_rows, max_rows, slot, ns, kv->k,      \
               kv->v, kv->k_scale, kv->v_scale)
  if (kv->dtype == ADEPT_KV_FP8) {
    if (dt == ADEPT_F32) ADEPT_STORE(float, true); else ADEPT_STORE(bf16, true);
  } else {
    if (dt == ADEPT_F32) ADEPT_STORE(float, false); else ADEPT_STORE(bf16, false);
  }
#undef ADEPT_STORE
  return launch_status("paged_store");
}

extern "C" adept_status adept_paged_load(adept_dtype dt, const adept_paged_kv* kv,
                                         const int32_t* slot, const int32_t* n_rows, int max_rows,
                                         void* k, int64_t k_stride, void* v, int64_t v_stride,
                                         void* stream) {
  ADEPT_TRY(check_rows("paged_load", dt, kv, k, k_stride, v, v_stride, max_rows, slot));
  if (max_rows == 0) return ADEPT_OK;
  const dim3 grid = row_grid(*kv, max_rows);
  const int H = kv->n_kv_heads, hd = kv->head_dim, ns = (int)paged_slots(*kv);
  hipStream_t s = as_stream(stream);
#define ADEPT_LOAD(T, FP8)                                                                     \
  ADEPT_LAUNCH((paged_load_kernel<T, FP8>), grid, dim3(kThreads), 0, s, H, hd, kv->k, kv->v,   \
               kv->k_scale, kv->v_scale, slot, n_rows, max_rows, ns, (T*)k, k_stride, (T*)v,   \
               v_stride)
  if (kv->dtype == ADEPT_KV_FP8) {
    if (dt == ADEPT_F32) ADEPT_LOAD(float, true); else ADEPT_LOAD(bf16, true);
  } else {
    if (dt == ADEPT_F32) ADEPT_LOAD(float, false); else ADEPT_LOAD(bf16, false);
  }
#undef ADEPT_LOAD
  return launch_status("paged_load");
}
