// Drafted tokens verified against the model's probabilities (adept_verify_drafts).
//
// With p_i = softmax(target row i / T) and q_i = softmax(draft row i / T), draft i
// is kept while u_i q_i(x_i) < p_i(x_i); the first one that is not is replaced by a
// token drawn from max(p_i - q_i, 0), normalised, and if all are kept one more is
// drawn from the row behind them.  So every emitted token is distributed as p.
//
// A token is the border between two sums, so everything behind the logits is in 64
// bits: a weight exp((l - max) / T), the sums, the comparisons.  With sums off by 1e-7,
// as in 32 bits, one draw in some hundred from a flat row of 32000 tokens (3e-5 each)
// would come from the other side of its border.  The vector units take 64-bit products
// and sums at the rate of unpacked 32-bit ones, and one exponential is about 20 of them.
//
// Two kernels.  The first takes the maximum and the sum of every row, 1024 logits a
// wave: all of the traffic, each logit once.  The second has a few workgroups for each
// sequence: every one makes the decision for itself (some partial sums from L2, less
// than one more kernel costs), takes its share of what p - q holds, and the last of them
// draws the token, by the shares' sums and then inside one.  64 sequences x 8 drafts x
// 32000 logits, f32: 33 and 20 us (at best 31 and 18.5: 4.1 TB/s, and 73 % of the SIMDs'
// cycles for the exponentials, in the first; round trips to memory in the second), one
// sequence x 4: 3.8 and 11.7.
#include <algorithm>
#include <climits>

#include "common.h"

namespace adept {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRowPer = 16;                  // logits of a lane in the first kernel
constexpr int kChunk = 64 * kRowPer;         // of a wave
constexpr int kPer = 8;
constexpr int kTile = kThreads * kPer;       // tokens of a share in the second
constexpr int kBlock = 64;                   // drafts that are decided at once

// A chunk of a row, or a row: its maximum (NaN left out), that value's first index
// (where it is asked for) and the sum of the weights.
struct Part {
  double sum;
  float top;
  int at;
};
enum PickMode { kPickGreedy, kPickRow, kPickRest, kPickOthers };

template <typename T>
struct Verify {
  int n_seq, g, vocab, chunks, tiles, groups;   // groups: workgroups of a sequence
  const T* target;
  int64_t t_stride;
  const T* draft;               // nullable
  int64_t d_stride;
  const int32_t *tokens, *n_draft;
  const float *temperature, *u;
  int32_t *out, *kept;
  Part* part;                   // [n_seq (g + 1) target rows, n_seq g draft rows][chunks]
  uint64_t* rest;               // [n_seq][tiles], doubles
  unsigned* ticket;             // [n_seq]

  __device__ __forceinline__ int drafts(int b) const {
    return n_draft ? min(max(n_draft[b], 0), g) : g;
  }
  // log2(e) / T; 0 or less: the largest logit
  __device__ __forceinline__ double slope(int b, bool* greedy) const {
    const float t = temperature ? temperature[b] : 1.0f;
    *greedy = !(t > 0.0f);
    return *greedy ? 1.0 : 1.4426950408889634 / (double)t;
  }
  __device__ __forceinline__ const T* target_row(int b, int i) const {
    return target + ((int64_t)b * (g + 1) + i) * t_stride;
  }
  __device__ __forceinline__ const T* draft_row(int b, int i) const {
    return draft + ((int64_t)b * g + i) * d_stride;
  }
  __device__ __forceinline__ const Part* target_part(int b, int i) const {
    return part + ((int64_t)b * (g + 1) + i) * chunks;
  }
  __device__ __forceinline__ const Part* draft_part(int b, int i) const {
    return part + ((int64_t)n_seq * (g + 1) + (int64_t)b * g + i) * chunks;
  }
};

// How many logits a row's chunks start before the row, so that their vectors are
// aligned: chunk c holds the indices c kChunk - lead .. (c + 1) kChunk - lead - 1.
template <typename T>
__device__ __forceinline__ int lead_of(const T* row) {
  return (int)(((uintptr_t)row & 15) / sizeof(T));
}

// 2^x for x <= 0, 0 for NaN: 2^n 2^f with n = rint(x), and 2^f by the polynomial of
// degree 10 through the Chebyshev points of [-1/2, 1/2] (off by 3e-16 of it).  The
// first kernel is bound by these instructions: the coefficients are kept in scalar
// registers (as constants they took two moves for each product: 640 instructions a
// wave, now 390; 64 x 8 drafts of 32000 logits 38 us, now 33).
struct Exp2 {
  double c[10];
  __device__ __forceinline__ Exp2() {
    constexpr double k[10] = {0.69314718055995,      0.24022650695910097,   0.05550410866444772,
                              0.009618129107606888,  0.0013333558230164974, 0.0001540353044173605,
                              1.5252657260200837e-05, 1.321544258792169e-06, 1.0208690299958306e-07,
                              7.072585949269223e-09};
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      c[i] = k[i];
      asm("" : "+s"(c[i]));
    }
  }
  __device__ __forceinline__ double operator()(double x) const {
    x = fmax(x, -1100.0);   // 2^-1100 is 0
    const double n = rint(x), f = x - n;
    double s = c[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) s = fma(s, f, c[i]);
    return ldexp(fma(s, f, 1.0), (int)n);
  }
};

// The weight of a logit in a row whose largest is `top`, exp((l - top) / T): none for NaN
// and -inf; where the largest is +inf, the infinite ones share the row.
__device__ __forceinline__ double weight(const Exp2& exp2, float l, float top, double slope) {
  if (top == INFINITY) return l == INFINITY ? 1.0 : 0.0;   // uniform over a row
  return exp2(((double)l - (double)top) * slope);
}

// Scans over a wave by DPP moves: a shuffle through LDS is ten times the latency, and
// the second kernel is a chain of them.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_f64(double v) {   // 0 where there is no lane to read
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double lane_f64(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
constexpr int kShr = 0x110, kBcast15 = 0x142, kBcast31 = 0x143;   // row_shr, row_bcast
// the running sum up to and with a lane
__device__ __forceinline__ double scan_f64(double v) {
  v += dpp_f64<kShr + 1, 0xf>(v);
  v += dpp_f64<kShr + 2, 0xf>(v);
  v += dpp_f64<kShr + 4, 0xf>(v);
  v += dpp_f64<kShr + 8, 0xf>(v);
  v += dpp_f64<kBcast15, 0xa>(v);
  v += dpp_f64<kBcast31, 0xc>(v);
  return v;
}
__device__ __forceinline__ double sum_f64(double v) { return lane_f64(scan_f64(v), 63); }
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_f32(float v) {     // -inf where there is no lane to read
  return __uint_as_float(__builtin_amdgcn_update_dpp(0xff800000u, __float_as_uint(v), CTRL, ROWS, 0xf,
                                                     false));
}
__device__ __forceinline__ float max_f32(float v) {
  v = fmaxf(v, dpp_f32<kShr + 1, 0xf>(v));
  v = fmaxf(v, dpp_f32<kShr + 2, 0xf>(v));
  v = fmaxf(v, dpp_f32<kShr + 4, 0xf>(v));
  v = fmaxf(v, dpp_f32<kShr + 8, 0xf>(v));
  v = fmaxf(v, dpp_f32<kBcast15, 0xa>(v));
  v = fmaxf(v, dpp_f32<kBcast31, 0xc>(v));
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// Block sums, the same in every thread.
__device__ __forceinline__ double block_sum(double v, double* sh) {
  v = sum_f64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = sh[0];
  for (int w = 1; w < kWaves; ++w) s += sh[w];
  return s;
}

// Loads from global memory: a row chosen among two is a flat pointer otherwise, whose
// loads wait for each other.
__device__ __forceinline__ float load_one(const float* p) {
  return *(const __attribute__((address_space(1))) float*)(uintptr_t)p;
}
__device__ __forceinline__ float load_one(const bf16* p) {
  return bf2f(*(const __attribute__((address_space(1))) bf16*)(uintptr_t)p);
}
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) u32x4_t global_u32x4_t;
__device__ __forceinline__ void load_vec(const float* p, float* x) {
  const u32x4_t w = *(const global_u32x4_t*)(uintptr_t)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]);
}
__device__ __forceinline__ void load_vec(const bf16* p, float* x) {
  const u32x4_t u = *(const global_u32x4_t*)(uintptr_t)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(u[e] << 16);
    x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
  }
}

// The first index of the largest value over a wave.
__device__ __forceinline__ void wave_first_max(float& top, int& at) {
  for (int o = 32; o > 0; o >>= 1) {
    const float ot = __shfl_xor(top, o, 64);
    const int oa = __shfl_xor(at, o, 64);
    if (ot > top || (ot == top && oa < at)) { top = ot; at = oa; }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_rows_kernel(Verify<T> a, int rows) {
  constexpr int VEC = 16 / sizeof(T), J = kRowPer / VEC;
  const int lane = threadIdx.x & 63;
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6));
  const int rows_t = a.n_seq * (a.g + 1);
  const int r = unit / a.chunks, c = unit % a.chunks;
  if (r >= rows) return;
  const bool of_target = r < rows_t;
  const int per = of_target ? a.g + 1 : a.g, at_row = of_target ? r : r - rows_t;
  const int b = at_row / per, i = at_row % per;
  if (i >= a.drafts(b) + (of_target ? 1 : 0)) return;
  bool greedy;
  const double slope = a.slope(b, &greedy);
  if (of_target && i == 0 && c == 0 && lane == 0) a.ticket[b] = 0;
  if (greedy && !of_target) return;
  const T* row = of_target ? a.target_row(b, i) : a.draft_row(b, i);
  const int base = c * kChunk - lead_of(row);
  float x[kRowPer];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int v = base + (j * 64 + lane) * VEC;
    if (v >= 0 && v <= a.vocab - VEC) {
      load_vec(row + v, x + j * VEC);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        x[j * VEC + e] = v + e >= 0 && v + e < a.vocab ? load_one(row + v + e) : -INFINITY;
    }
  }
  float top = -INFINITY;
  int at = 0;
  double s = 0.0;
  if (greedy) {
    at = INT_MAX;
#pragma unroll
    for (int e = 0; e < kRowPer; ++e)
      if (x[e] > top) {
        top = x[e];
        at = base + (e / VEC * 64 + lane) * VEC + e % VEC;
      }
    wave_first_max(top, at);
  } else {
#pragma unroll
    for (int e = 0; e < kRowPer; ++e) top = fmaxf(top, x[e]);   // leaves NaN out
    top = max_f32(top);
    if (top > -INFINITY) {
      const Exp2 exp2;
      if (top == INFINITY) {
#pragma unroll
        for (int e = 0; e < kRowPer; ++e) s += x[e] == INFINITY ? 1.0 : 0.0;
      } else {
#pragma unroll
        for (int e = 0; e < kRowPer; ++e) s += exp2(((double)x[e] - (double)top) * slope);
      }
      s = sum_f64(s);
    }
  }
  if (lane == 0) a.part[(int64_t)r * a.chunks + c] = Part{s, top, at};
}

// A row's maximum (greedy: with its first index) and its sum, by one wave; own: the
// lane's first part, which first_part loads ahead.
__device__ __forceinline__ Part first_part(const Part* part, int chunks) {
  const int lane = threadIdx.x & 63;
  return lane < chunks ? part[lane] : Part{0.0, -INFINITY, INT_MAX};
}
__device__ __forceinline__ Part row_total(const Exp2& exp2, Part own, const Part* part, int chunks,
                                          double slope, bool greedy) {
  const int lane = threadIdx.x & 63;
  if (greedy) {
    for (int c = lane + 64; c < chunks; c += 64)
      if (part[c].top > own.top) own = part[c];
    wave_first_max(own.top, own.at);
    return own;
  }
  float top = own.top;
  for (int c = lane + 64; c < chunks; c += 64) top = fmaxf(top, part[c].top);
  top = max_f32(top);
  if (!(top > -INFINITY)) return Part{0.0, top, INT_MAX};
  double s = own.sum * weight(exp2, own.top, top, slope);
  for (int c = lane + 64; c < chunks; c += 64)
    s += part[c].sum * weight(exp2, part[c].top, top, slope);
  return Part{sum_f64(s), top, 0};
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_token_kernel(Verify<T> a) {
  __shared__ double sh[kWaves];
  __shared__ Part pt[kBlock], qt[kBlock];
  __shared__ Part p_row;
  __shared__ int first, firsts[kWaves], lasts[kWaves];
  __shared__ bool is_last;
  const int b = blockIdx.x / a.groups, group = blockIdx.x % a.groups;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = a.drafts(b);
  const Exp2 exp2;
  bool greedy;
  const double slope = a.slope(b, &greedy);
  const float u_last = a.u[(int64_t)b * (a.g + 1) + a.g];

  // the first draft that is not kept
  int kept = n;
  Part q{0.0, 0.0f, 0};
  for (int i0 = 0; i0 < n; i0 += kBlock) {
    const int m = min(n - i0, kBlock);
    // wave 0, lane i: draft i0 + i
    float lp = -INFINITY, lq = -INFINITY, u = 0.0f;
    int x = -1;
    if (tid < m) {
      x = a.tokens[(int64_t)b * a.g + i0 + tid];
      u = a.u[(int64_t)b * (a.g + 1) + i0 + tid];
      if (x < 0 || x >= a.vocab) x = -1;
      if (x >= 0 && !greedy) {
        lp = ld(a.target_row(b, i0 + tid) + x);
        if (a.draft) lq = ld(a.draft_row(b, i0 + tid) + x);
      }
    }
    // two drafts of a wave at a time, their parts loaded together
    const bool drawn = a.draft && !greedy;
    for (int i = wave; i < m; i += 2 * kWaves) {
      Part pf[2], qf[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = i0 + min(i + j * kWaves, m - 1);
        pf[j] = first_part(a.target_part(b, row), a.chunks);
        if (drawn) qf[j] = first_part(a.draft_part(b, row), a.chunks);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int k = i + j * kWaves;
        if (k >= m) break;
        const Part p = row_total(exp2, pf[j], a.target_part(b, i0 + k), a.chunks, slope, greedy);
        Part r{0.0, 0.0f, 0};
        if (drawn) r = row_total(exp2, qf[j], a.draft_part(b, i0 + k), a.chunks, slope, false);
        if (lane == 0) {
          pt[k] = p;
          qt[k] = r;
        }
      }
    }
    __syncthreads();
    if (wave == 0) {
      bool keep = true;
      if (lane < m) {
        const Part p = pt[lane], r = qt[lane];
        if (greedy) {
          keep = x >= 0 && x == p.at;
        } else {
          const double px = x >= 0 && p.sum > 0.0 ? weight(exp2, lp, p.top, slope) / p.sum : 0.0;
          const double qx = !a.draft ? 1.0
                            : x >= 0 && r.sum > 0.0 ? weight(exp2, lq, r.top, slope) / r.sum : 0.0;
          keep = (double)u * qx < px;
        }
      }
      const uint64_t no = __ballot(!keep);
      if (lane == 0) first = no ? __ffsll((unsigned long long)no) - 1 : m;
    }
    __syncthreads();
    const int f = first;
    if (f < m) {
      kept = i0 + f;
      q = qt[f];
      if (tid == 0) p_row = pt[f];
      break;
    }
    __syncthreads();
  }
  if (kept == n && wave == 0) {
    const Part* part = a.target_part(b, n);
    const Part p = row_total(exp2, first_part(part, a.chunks), part, a.chunks, slope, greedy);
    if (lane == 0) p_row = p;
  }
  __syncthreads();
  const Part p = p_row;
  int mode = greedy ? kPickGreedy : kept == n ? kPickRow : a.draft ? kPickRest : kPickOthers;
  if (mode == kPickRest && !(q.sum > 0.0)) mode = kPickRow;
  if (!greedy && !(p.sum > 0.0)) mode = kPickGreedy;   // no distribution: p.at is no token
  if (mode != kPickRest && group != 0) return;

  const T* row = a.target_row(b, kept);
  const T* other = mode == kPickRest ? a.draft_row(b, kept) : row;
  int gone = mode == kPickOthers ? a.tokens[(int64_t)b * a.g + kept] : -1;
  const double ip = mode == kPickRest ? 1.0 / p.sum : 1.0, iq = mode == kPickRest ? 1.0 / q.sum : 0.0;
  // the logits of token v, in one batch with others', and what it holds in this mode
  auto load = [&](int v, float& l, float& o) {
    const int at = min(max(v, 0), a.vocab - 1);
    l = load_one(row + at);
    o = mode == kPickRest ? load_one(other + at) : 0.0f;
  };
  auto held = [&](int v, float l, float o) {
    if (v < 0 || v >= a.vocab || v == gone) return 0.0;
    const double w = weight(exp2, l, p.top, slope);
    if (mode != kPickRest) return w;
    // what is within the rounding of the rows' sums is none: of equal rows nothing is left
    const double pv = w * ip, d = pv - weight(exp2, o, q.top, slope) * iq;
    return d > pv * 0x1p-40 ? d : 0.0;
  };
  if (mode == kPickRest) {
    // The shares' sums meet by device-scope atomics, so no cache has to be written back in
    // between; a workgroup counts itself once its atomics have returned, so the one that
    // counts last finds every sum (with fences instead 84 us at 64 sequences).
    uint64_t seen = 0;
    for (int t = group; t < a.tiles; t += a.groups) {
      double s = 0.0;
      float l[kPer], o[kPer];
#pragma unroll
      for (int j = 0; j < kPer; ++j) load(t * kTile + j * kThreads + tid, l[j], o[j]);
#pragma unroll
      for (int j = 0; j < kPer; ++j) s += held(t * kTile + j * kThreads + tid, l[j], o[j]);
      s = block_sum(s, sh);
      if (tid == 0)
        seen |= __hip_atomic_exchange(&a.rest[(int64_t)b * a.tiles + t], __builtin_bit_cast(uint64_t, s),
                                      __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (tid == 0) {
      unsigned one = 1;
      asm volatile("" : "+v"(one) : "v"(seen));   // counted after the sums are there
      is_last = __hip_atomic_fetch_add(&a.ticket[b], one, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT) == (unsigned)a.groups - 1;
      asm volatile("" ::: "memory");
    }
    __syncthreads();
    if (!is_last) return;
  }

  int next = -1;
  if (mode == kPickGreedy) {
    if (greedy && p.at != INT_MAX) next = p.at;
  } else {
    // parts of the row that are searched: shares, or the first kernel's chunks
    const Part* part = a.target_part(b, kept);
    const int lead = lead_of(row);
    double whole_gone = 0.0;              // kPickOthers: the chunk of the token left out
    int c_gone = gone >= 0 && gone < a.vocab ? (gone + lead) / kChunk : -1;
    if (c_gone >= 0) {
      double s = 0.0;
      for (int j = tid; j < kChunk; j += kThreads) {
        const int v = c_gone * kChunk - lead + j;
        float l, o;
        load(v, l, o);
        s += held(v, l, o);
      }
      whole_gone = block_sum(s, sh);
    }
    auto mass = [&](int c) {
      if (mode == kPickRest) {
        if (c >= a.tiles) return 0.0;
        return __builtin_bit_cast(double, __hip_atomic_load(&a.rest[(int64_t)b * a.tiles + c],
                                                            __ATOMIC_RELAXED,
                                                            __HIP_MEMORY_SCOPE_AGENT));
      }
      if (c >= a.chunks) return 0.0;
      if (c == c_gone) return whole_gone;
      return part[c].top > -INFINITY ? part[c].sum * weight(exp2, part[c].top, p.top, slope) : 0.0;
    };
    int parts = mode == kPickRest ? a.tiles : a.chunks;
    auto whole = [&]() {
      double s = 0.0;
      for (int c = lane; c < parts; c += 64) s += mass(c);
      return sum_f64(s);
    };
    double total = whole();
    if (mode != kPickRow && !(total > 0.0)) {   // p is q: nothing is left of it
      mode = kPickRow;
      parts = a.chunks;
      gone = c_gone = -1;
      total = p.sum;
    }
    const double aim = u_last > 0.0f ? (double)u_last * total : 0.0;
    double run = 0.0, before = 0.0;       // before: the sum of the parts before `hit`
    int found_part = -1;
    for (int c0 = 0; c0 < parts; c0 += 64) {   // every wave for itself
      const double m = mass(c0 + lane);
      const double s = scan_f64(m);
      // the part that passes the aim, else the last one that holds something
      const uint64_t over = __ballot(m > 0.0 && run + s > aim);
      const uint64_t some = __ballot(m > 0.0);
      const int hit = over ? __ffsll((unsigned long long)over) - 1
                           : some ? 63 - __clzll((long long)some) : -1;
      if (hit >= 0) {
        found_part = c0 + hit;
        before = run + lane_f64(s - m, hit);
      }
      if (over) break;
      run += lane_f64(s, 63);
    }
    if (found_part >= 0) {
      const int size = mode == kPickRest ? kTile : kChunk;
      const int lo = found_part * size - (mode == kPickRest ? 0 : lead);
      double w[kPer], s = 0.0;
      float l[kPer], o[kPer];
#pragma unroll
      for (int e = 0; e < kPer; ++e) load(lo + tid * kPer + e, l[e], o[e]);
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int j = tid * kPer + e;
        w[e] = j < size ? held(lo + j, l[e], o[e]) : 0.0;
        s += w[e];
      }
      const double scan = scan_f64(s);
      __syncthreads();
      if (lane == 63) sh[wave] = scan;
      __syncthreads();
      double at = before + (scan - s);
      for (int v = 0; v < wave; ++v) at += sh[v];
      int hit = INT_MAX, last = -1;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        at += w[e];
        if (w[e] > 0.0) {
          if (at > aim) hit = min(hit, lo + tid * kPer + e);
          last = lo + tid * kPer + e;
        }
      }
      // indices ascend with the lanes
      const uint64_t hits = __ballot(hit != INT_MAX), some = __ballot(last >= 0);
      hit = hits ? __builtin_amdgcn_readlane(hit, __ffsll((unsigned long long)hits) - 1) : INT_MAX;
      last = some ? __builtin_amdgcn_readlane(last, 63 - __clzll((long long)some)) : -1;
      if (lane == 0) {
        firsts[wave] = hit;
        lasts[wave] = last;
      }
      __syncthreads();
      for (int v = 0; v < kWaves; ++v) {
        hit = min(hit, firsts[v]);
        last = max(last, lasts[v]);
      }
      next = hit != INT_MAX ? hit : last;
    }
  }
  for (int i = tid; i <= a.g; i += kThreads)
    a.out[(int64_t)b * (a.g + 1) + i] =
        i < kept ? a.tokens[(int64_t)b * a.g + i] : i == kept ? next : -1;
  if (tid == 0) a.kept[b] = kept;
}

int chunks_of(int vocab) { return ceil_div((long)vocab + 7, kChunk); }   // 7: the largest lead
int tiles_of(int vocab) { return ceil_div(vocab, kTile); }
struct VerifyWs {
  size_t rest, ticket, total;
};
VerifyWs verify_ws(int64_t n_seq, int64_t g, int vocab) {
  auto align = [](size_t x) { return (x + 255) / 256 * 256; };
  VerifyWs w{};
  w.rest = align((size_t)(n_seq * (2 * g + 1) * chunks_of(vocab)) * sizeof(Part));
  w.ticket = w.rest + align((size_t)(n_seq * tiles_of(vocab)) * sizeof(uint64_t));
  w.total = w.ticket + align((size_t)n_seq * sizeof(unsigned));
  return w;
}

template <typename T>
adept_status verify_launch(Verify<T> a, void* workspace, hipStream_t s) {
  const VerifyWs w = verify_ws(a.n_seq, a.g, a.vocab);
  a.chunks = chunks_of(a.vocab);
  a.tiles = tiles_of(a.vocab);
  a.part = (Part*)workspace;
  a.rest = (uint64_t*)((char*)workspace + w.rest);
  a.ticket = (unsigned*)((char*)workspace + w.ticket);
  const int rows = a.n_seq * (a.g + 1) + (a.draft ? a.n_seq * a.g : 0);
  // one wave a workgroup while that spreads them over the chip's CUs
  const int units = rows * a.chunks, waves = units >= 4096 ? kWaves : 1;
  ADEPT_LAUNCH(verify_rows_kernel<T>, dim3(ceil_div(units, waves)), dim3(64 * waves), 0, s, a, rows);
  ADEPT_CHECK_LAUNCH("verify_rows");
  // shares only where something can be left of p - q; about 1024 workgroups at most
  a.groups = a.draft ? std::min(a.tiles, std::max(1, 1024 / a.n_seq)) : 1;
  ADEPT_LAUNCH(verify_token_kernel<T>, dim3((unsigned)a.n_seq * a.groups), dim3(kThreads), 0, s, a);
  return launch_status("verify_token");
}

}  // namespace
}  // namespace adept

using namespace adept;

extern "C" size_t adept_verify_drafts_workspace_bytes(int n_seq, int max_draft, int vocab) {
  if (n_seq <= 0 || max_draft < 0 || vocab <= 0) return 0;
  return verify_ws(n_seq, max_draft, vocab).total;
}

extern "C" adept_status adept_verify_drafts(adept_dtype dt, int n_seq, int max_draft, int vocab,
                                            const void* target, int64_t target_stride,
                                            const void* draft, int64_t draft_stride,
                                            const int32_t* tokens, const int32_t* n_draft,
                                            const float* temperature, const float* u,
                                            int32_t* out_tokens, int32_t* n_kept, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  ADEPT_REQUIRE(dt == ADEPT_F32 || dt == ADEPT_BF16, "verify_drafts: bad dtype");
  ADEPT_REQUIRE(n_seq >= 0 && max_draft >= 0 && vocab > 0 && vocab <= INT_MAX - kChunk,
                "verify_drafts: bad sizes");
  if (n_seq == 0) return ADEPT_OK;
  ADEPT_REQUIRE((int64_t)n_seq * (2 * (int64_t)max_draft + 1) * chunks_of(vocab) < 1 << 24,
                "verify_drafts: too many logits for a call");   // a grid's bound
  ADEPT_REQUIRE(target && u && out_tokens && n_kept && (tokens || max_draft == 0),
                "verify_drafts: NULL tensor");
  const uintptr_t esz = dt == ADEPT_F32 ? 4 : 2;
  ADEPT_REQUIRE((uintptr_t)target % esz == 0 && (uintptr_t)draft % esz == 0,
                "verify_drafts: logits must be aligned to their type");
  ADEPT_REQUIRE(target_stride >= vocab && (!draft || max_draft == 0 || draft_stride >= vocab),
                "verify_drafts: rows shorter than the vocabulary");
  const size_t need = verify_ws(n_seq, max_draft, vocab).total;
  if (!workspace || workspace_bytes < need || !aligned16(workspace)) {
    set_error("verify_drafts: a 16-byte aligned workspace of %zu bytes needed", need);
    return ADEPT_E_WORKSPACE;
  }
  hipStream_t s = as_stream(stream);
  auto fill = [&](auto a) {
    typedef decltype(a.target) P;
    a.n_seq = n_seq; a.g = max_draft; a.vocab = vocab;
    a.target = (P)target; a.t_stride = target_stride;
    a.draft = max_draft ? (P)draft : nullptr; a.d_stride = draft_stride;
    a.tokens = tokens; a.n_draft = n_draft; a.temperature = temperature; a.u = u;
    a.out = out_tokens; a.kept = n_kept;
    return verify_launch(a, workspace, s);
  };
  return dt == ADEPT_F32 ? fill(Verify<float>{}) : fill(Verify<bf16>{});
}
