// Weights in 4 bits (quant.h): packed from a matrix, read back, and the product of
// few rows with them (the few-row GEMM of gemm_direct.hip over the packed form).
//
// Packing and reading back: one wave for a block of 16 rows and 128 of K.  Packing
// reads whole lines of the rows and turns the codes in LDS into the block's order.
// Bound by the HBM traffic of the source, which passes by non-temporal loads: 11008 x
// 4096 bf16 packed in 24 us (4.8 TB/s; 32 with ordinary ones), read back in 20.
#include <climits>

#include "quant.h"

namespace adept {
namespace {

constexpr int kWaves = 4;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void load8(const float* p, bool whole, int left, float (&x)[8]) {
  if (whole) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const u32x4_t w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + i));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i + e] = __uint_as_float(w[e]);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = e < left ? p[e] : 0.0f;
}
__device__ __forceinline__ void load8(const bf16* p, bool whole, int left, float (&x)[8]) {
  if (whole) {
    const u32x4_t u = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(u[e] << 16);
      x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = e < left ? bf2f(p[e]) : 0.0f;
}

// w [n][k], rows ldw elements apart, any alignment.
template <typename T>
__global__ __launch_bounds__(64 * kWaves) void quant_pack_kernel(int n, int k, const T* __restrict__ w,
                                                                 int64_t ldw, int kb, int64_t blocks,
                                                                 uint8_t* __restrict__ codes,
                                                                 uint8_t* __restrict__ scales) {
  __shared__ __attribute__((aligned(16))) uint32_t turn[kWaves][kQuantBlock / 4];
  __shared__ __attribute__((aligned(4))) uint8_t bytes[kWaves][kQuantScales];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t blk = (int64_t)blockIdx.x * kWaves + wave;
  if (blk < blocks) {
    const int64_t row0 = blk / kb * kQuantRows;
    // a lane has eight of the 128 k of rows lane / 16 + 4 i, a group is four lanes
    const int chunk = lane & 15, k0 = (int)(blk % kb) * kQuantK + 8 * chunk;
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = row0 + 4 * i + (lane >> 4);
      const int left = row < n ? min(max(k - k0, 0), 8) : 0;
      const T* p = w + (left > 0 ? row * ldw + k0 : 0);
      load8(p, left == 8 && ((uintptr_t)p & 15) == 0, left, x[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[i][e]) & 0x7fffffffu);
      top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
      top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
      // top = m 2^x, 1 <= m < 2: the least E with top <= 7 2^E = 1.75 2^(E + 2)
      int b = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
      b = min(max(b, kQuantScaleMin), kQuantScaleMax);
      const float inv = __uint_as_float((uint32_t)(254 - b) << 23);
      const bool fine = top < 0x7f800000u;
      if (!fine) b = kQuantScaleNan;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = fine ? x[i][e] * inv : 0.0f;   // exact, or far below 1/4
      // to the nearest code, ties to even, at most 6
      uint32_t c = 0;
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], 1.0f, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.0f, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.0f, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.0f, 3);
      const int r16 = 4 * i + (lane >> 4), h = chunk >> 2, q = chunk & 3;
      turn[wave][(r16 + 16 * q) * 4 + h] = c;
      if (q == 0) bytes[wave][r16 * 4 + h] = (uint8_t)b;
    }
  }
  __syncthreads();
  if (blk >= blocks) return;
  *reinterpret_cast<uint4*>(codes + blk * kQuantBlock + lane * 16) =
      *reinterpret_cast<const uint4*>(&turn[wave][lane * 4]);
  if (lane < kQuantScales / 4)
    *reinterpret_cast<uint32_t*>(scales + blk * kQuantScales + lane * 4) =
        *reinterpret_cast<const uint32_t*>(&bytes[wave][lane * 4]);
}

template <typename T>
__global__ __launch_bounds__(64 * kWaves) void quant_unpack_kernel(
    int n, int k, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int kb,
    int64_t blocks, T* __restrict__ w, int64_t ldw) {
  const int64_t blk = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (blk >= blocks) return;
  const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
  const int64_t row = blk / kb * kQuantRows + r16;
  if (row >= n) return;
  const int k0 = (int)(blk % kb) * kQuantK + 8 * q;
  const uint4 c = *reinterpret_cast<const uint4*>(codes + blk * kQuantBlock + lane * 16);
  const uint32_t cw[4] = {c.x, c.y, c.z, c.w};
  const uint32_t bytes = *reinterpret_cast<const uint32_t*>(scales + blk * kQuantScales + r16 * 4);
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int left = min(k - k0 - 32 * h, 8);
    if (left <= 0) break;
    const uint4 v = __builtin_bit_cast(uint4, quant_expand(cw[h], bytes >> (8 * h)));
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
    T* p = w + row * ldw + k0 + 32 * h;
    if constexpr (sizeof(T) == 2) {
      if (left == 8 && ((uintptr_t)p & 15) == 0) {
        *reinterpret_cast<uint4*>(p) = v;
        continue;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) st(p + e, __uint_as_float(e & 1 ? u[e >> 1] & 0xffff0000u : u[e >> 1] << 16));
  }
}

adept_status check_matrix(const char* what, int n, int k, const void* codes, const void* scales) {
  ADEPT_REQUIRE(n > 0 && k > 0 && n <= INT_MAX - kQuantRows && k <= 1 << 29,
                "%s: bad sizes", what);
  ADEPT_REQUIRE(quant_blocks(n, k) <= (int64_t)kWaves << 23, "%s: a matrix of %d x %d is too large",
                what, n, k);   // a grid's bound
  ADEPT_REQUIRE(codes && scales && aligned16(codes) && aligned16(scales),
                "%s: codes and scales must be 16-byte aligned", what);
  return ADEPT_OK;
}

// Rows of a product with n weight rows: a grid's bound, of workgroups of up to 1024 threads.
adept_status check_rows(const char* what, int n, int max_rows) {
  ADEPT_REQUIRE(max_rows >= 0 && max_rows <= 64 * 65535 &&
                    (ceil_div(n, 16) + 7ll) * ceil_div(max_rows, 16) < 1 << 22,
                "%s: bad max_rows %d", what, max_rows);
  return ADEPT_OK;
}

}  // namespace
}  // namespace adept

using namespace adept;

extern "C" size_t adept_quant_codes_bytes(int n, int k) {
  return n > 0 && k > 0 ? (size_t)quant_blocks(n, k) * kQuantBlock : 0;
}

extern "C" size_t adept_quant_scales_bytes(int n, int k) {
  return n > 0 && k > 0 ? (size_t)quant_blocks(n, k) * kQuantScales : 0;
}

extern "C" adept_status adept_quant_pack(adept_dtype dt, int n, int k, const void* w, int64_t ldw,
                                         void* codes, void* scales, void* stream) {
  ADEPT_REQUIRE(dt == ADEPT_F32 || dt == ADEPT_BF16, "quant_pack: bad dtype");
  ADEPT_TRY(check_matrix("quant_pack", n, k, codes, scales));
  ADEPT_REQUIRE(w && (uintptr_t)w % (dt == ADEPT_F32 ? 4 : 2) == 0 && ldw >= k, "quant_pack: bad matrix");
  const int64_t blocks = quant_blocks(n, k);
  const dim3 grid((unsigned)((blocks + kWaves - 1) / kWaves)), block(64 * kWaves);
  const int kb = ceil_div(k, kQuantK);
  if (dt == ADEPT_F32)
    ADEPT_LAUNCH(quant_pack_kernel<float>, grid, block, 0, as_stream(stream), n, k, (const float*)w,
                 ldw, kb, blocks, (uint8_t*)codes, (uint8_t*)scales);
  else
    ADEPT_LAUNCH(quant_pack_kernel<bf16>, grid, block, 0, as_stream(stream), n, k, (const bf16*)w,
                 ldw, kb, blocks, (uint8_t*)codes, (uint8_t*)scales);
  return launch_status("quant_pack");
}

extern "C" adept_status adept_quant_unpack(adept_dtype dt, int n, int k, const void* codes,
                                           const void* scales, void* w, int64_t ldw, void* stream) {
  ADEPT_REQUIRE(dt == ADEPT_F32 || dt == ADEPT_BF16, "quant_unpack: bad dtype");
  ADEPT_TRY(check_matrix("quant_unpack", n, k, codes, scales));
  ADEPT_REQUIRE(w && (uintptr_t)w % (dt == ADEPT_F32 ? 4 : 2) == 0 && ldw >= k, "quant_unpack: bad matrix");
  const int64_t blocks = quant_blocks(n, k);
  const dim3 grid((unsigned)((blocks + kWaves - 1) / kWaves)), block(64 * kWaves);
  const int kb = ceil_div(k, kQuantK);
  if (dt == ADEPT_F32)
    ADEPT_LAUNCH(quant_unpack_kernel<float>, grid, block, 0, as_stream(stream), n, k,
                 (const uint8_t*)codes, (const uint8_t*)scales, kb, blocks, (float*)w, ldw);
  else
    ADEPT_LAUNCH(quant_unpack_kernel<bf16>, grid, block, 0, as_stream(stream), n, k,
                 (const uint8_t*)codes, (const uint8_t*)scales, kb, blocks, (bf16*)w, ldw);
  return launch_status("quant_unpack");
}

extern "C" adept_status adept_quant_linear(int n, int k, const void* x, int64_t x_stride,
                                           const int32_t* rows, const int32_t* n_rows, int max_rows,
                                           const void* codes, const void* scales, const void* bias,
                                           adept_dtype out_dt, void* y, int64_t y_stride,
                                           void* stream) {
  ADEPT_REQUIRE(out_dt == ADEPT_F32 || out_dt == ADEPT_BF16, "quant_linear: bad dtype");
  ADEPT_TRY(check_matrix("quant_linear", n, k, codes, scales));
  ADEPT_REQUIRE(k % 8 == 0, "quant_linear: k = %d is no multiple of 8", k);
  ADEPT_TRY(check_rows("quant_linear", n, max_rows));
  if (max_rows == 0) return ADEPT_OK;
  ADEPT_REQUIRE(x && y && aligned16(x) && x_stride >= k && x_stride % 8 == 0,
                "quant_linear: x must be 16-byte aligned rows, a multiple of 16 bytes apart");
  ADEPT_REQUIRE(y_stride >= n && (uintptr_t)y % (out_dt == ADEPT_F32 ? 4 : 2) == 0 &&
                    (uintptr_t)bias % 2 == 0,
                "quant_linear: bad output or bias");
  GemmArgs g{};
  g.M_max = max_rows; g.M_dev = n_rows; g.N = n; g.K = k;
  g.A = x; g.a_rows = rows; g.lda = x_stride; g.epi = EPI_STORE;
  g.C = y; g.ldc = y_stride; g.c_f32 = out_dt == ADEPT_F32; g.bias = bias; g.name = "quant_linear";
  g.quant = QuantView{(const uint8_t*)codes, (const uint8_t*)scales, nullptr, nullptr, 0, 0};
  return gemm_direct(g, as_stream(stream));
}

extern "C" adept_status adept_final_logits_quant(int d_model, int vocab, float eps,
                                                 const void* h0_buf, const void* h1_buf,
                                                 const int32_t* exit_layer, const int32_t* rows,
                                                 const int32_t* n_rows, int max_rows,
                                                 const void* norm_gain, const void* norm_bias,
                                                 const void* codes, const void* scales, void* x_norm,
                                                 float* logits, void* stream) {
  ADEPT_REQUIRE(d_model % 8 == 0, "final_logits_quant: bad sizes");
  ADEPT_REQUIRE(h0_buf && h1_buf && exit_layer && rows && norm_gain && x_norm && logits,
                "final_logits_quant: NULL tensor");
  ADEPT_TRY(check_matrix("final_logits_quant", vocab, d_model, codes, scales));
  ADEPT_TRY(check_rows("final_logits_quant", vocab, max_rows));
  ADEPT_REQUIRE(aligned16(h0_buf) && aligned16(h1_buf) && aligned16(x_norm) && aligned16(logits) &&
                    aligned16(norm_gain) && aligned16(norm_bias),
                "final_logits_quant: tensors must be 16-byte aligned");
  if (max_rows == 0) return ADEPT_OK;
  hipStream_t s = as_stream(stream);
  if (norm_bias)
    ADEPT_TRY(layernorm_rows_sel(ADEPT_BF16, d_model, eps, h0_buf, h1_buf, exit_layer, rows, n_rows,
                                 max_rows, norm_gain, norm_bias, x_norm, s));
  else
    ADEPT_TRY(rmsnorm_rows_sel(ADEPT_BF16, d_model, eps, h0_buf, h1_buf, exit_layer, rows, n_rows,
                               max_rows, norm_gain, x_norm, s));
  return adept_quant_linear(vocab, d_model, x_norm, d_model, nullptr, n_rows, max_rows, codes, scales,
                            nullptr, ADEPT_F32, logits, vocab, stream);
}
