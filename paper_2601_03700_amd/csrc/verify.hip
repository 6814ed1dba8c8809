// Drafted tokens verified against the model's probabilities (adept_verify_drafts).
//
// With p_i = softmax(target row i / T) and q_i = softmax(draft row i / T), draft i
// is kept while u_i q_i(x_i) < p_i(x_i); the first one that is not is replaced by a
// token drawn from max(p_i - q_i, 0), normalised, and if all are kept one more is
// drawn from the row behind them.  So every emitted token is distributed as p.
//
// A token is the border between two sums, so everything behind the logits is in 64
// bits: a weight exp((l - max) / T), the sums, the comparisons.  In 32 bits one
// token in a few thousand of a flat row of 32000 came from the other side of its
// border.  The vector units take 64-bit products and sums at the rate of unpacked
// 32-bit ones, and one exponential is about 20 of them.
//
// Three kernels: the maximum and the sum of every row's chunks (all of the traffic:
// the logits once); the decision of each sequence, and what the row of its next
// token holds, chunk by chunk; the token itself, by the chunks' sums and then inside
// one chunk.
#include <climits>

#include "common.h"

namespace adept {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                      // logits of a thread
constexpr int kChunk = kThreads * kPer;

// A chunk of a row: its maximum (NaN left out), that value's first index, and the
// sum of exp((l - max) / T).
struct Part {
  double sum;
  float top;
  int at;
};
enum PickMode { kPickGreedy, kPickRow, kPickRest, kPickOthers };
// What the next token of a sequence is drawn from.
struct Pick {
  double p_total, q_total;
  float p_top, q_top;
  int kept, mode, at, gone;   // at: the greedy token; gone: the token left out (kPickOthers)
};

template <typename T>
struct Verify {
  int n_seq, g, vocab, chunks;
  const T* target;
  int64_t t_stride;
  const T* draft;               // nullable
  int64_t d_stride;
  const int32_t *tokens, *n_draft;
  const float *temperature, *u;
  int32_t *out, *kept;
  Part* part;                   // [n_seq (g + 1) target rows, n_seq g draft rows][chunks]
  double* rest;                 // [n_seq][chunks]
  Pick* pick;                   // [n_seq]

  __device__ __forceinline__ int drafts(int b) const {
    return n_draft ? min(max(n_draft[b], 0), g) : g;
  }
  // 1 / T; 0 or less: the largest logit
  __device__ __forceinline__ double inverse(int b, bool* greedy) const {
    const float t = temperature ? temperature[b] : 1.0f;
    *greedy = !(t > 0.0f);
    return *greedy ? 1.0 : 1.0 / (double)t;
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

// e^x for x <= 0: x = n ln 2 + r, |r| <= ln 2 / 2, and the series of e^r up to r^12
// (what is left out is below 2e-16 of it).
__device__ __forceinline__ double exp_neg(double x) {
  if (x < -745.0) return 0.0;
  const double n = rint(x * 1.4426950408889634);
  double r = fma(n, -0.6931471805599453, x);
  r = fma(n, -2.3190468138462996e-17, r);      // ln 2 less its 64-bit value
  double s = 1.0 / 479001600.0;
  s = fma(s, r, 1.0 / 39916800.0);
  s = fma(s, r, 1.0 / 3628800.0);
  s = fma(s, r, 1.0 / 362880.0);
  s = fma(s, r, 1.0 / 40320.0);
  s = fma(s, r, 1.0 / 5040.0);
  s = fma(s, r, 1.0 / 720.0);
  s = fma(s, r, 1.0 / 120.0);
  s = fma(s, r, 1.0 / 24.0);
  s = fma(s, r, 1.0 / 6.0);
  s = fma(s, r, 0.5);
  s = fma(s, r, 1.0);
  s = fma(s, r, 1.0);
  return ldexp(s, (int)n);
}

// The weight of a logit in a row whose largest is `top`: none for NaN and -inf; where
// the largest is +inf, the infinite ones share the row.
__device__ __forceinline__ double weight(float l, float top, double inv) {
  if (!(l > -INFINITY)) return 0.0;
  if (top == INFINITY) return l == INFINITY ? 1.0 : 0.0;
  return exp_neg(((double)l - (double)top) * inv);
}

// Block sums, the same in every thread.
__device__ __forceinline__ double block_sum(double v, double* sh) {
  v = wave_sum_f64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = sh[0];
  for (int w = 1; w < kThreads / 64; ++w) s += sh[w];
  return s;
}

__device__ __forceinline__ void load_vec(const float* p, float (&x)[4]) {
  const float4 w = *reinterpret_cast<const float4*>(p);
  x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
}
__device__ __forceinline__ void load_vec(const bf16* p, float (&x)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(u[e] << 16);
    x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_rows_kernel(Verify<T> a) {
  constexpr int VEC = 16 / sizeof(T), J = kPer / VEC;
  __shared__ double sh[kThreads / 64];
  __shared__ float tops[kThreads / 64];
  __shared__ int ats[kThreads / 64];
  const int rows_t = a.n_seq * (a.g + 1);
  const int r = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks;
  const bool of_target = r < rows_t;
  const int per = of_target ? a.g + 1 : a.g;
  const int b = (of_target ? r : r - rows_t) / per, i = (of_target ? r : r - rows_t) % per;
  if (i >= a.drafts(b) + (of_target ? 1 : 0)) return;
  bool greedy;
  const double inv = a.inverse(b, &greedy);
  if (greedy && !of_target) return;
  const T* row = of_target ? a.target_row(b, i) : a.draft_row(b, i);
  const int base = c * kChunk - lead_of(row);
  float x[J][VEC];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int v = base + (j * kThreads + (int)threadIdx.x) * VEC;
    if (v >= 0 && v <= a.vocab - VEC) {
      load_vec(row + v, x[j]);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        x[j][e] = v + e >= 0 && v + e < a.vocab ? ld(row + v + e) : -INFINITY;
    }
  }
  float top = -INFINITY;
  int at = INT_MAX;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (x[j][e] > top) {
        top = x[j][e];
        at = base + (j * kThreads + (int)threadIdx.x) * VEC + e;
      }
  for (int o = 32; o > 0; o >>= 1) {
    const float ot = __shfl_xor(top, o, 64);
    const int oa = __shfl_xor(at, o, 64);
    if (ot > top || (ot == top && oa < at)) { top = ot; at = oa; }
  }
  if ((threadIdx.x & 63) == 0) {
    tops[threadIdx.x >> 6] = top;
    ats[threadIdx.x >> 6] = at;
  }
  __syncthreads();
  top = tops[0];
  at = ats[0];
  for (int w = 1; w < kThreads / 64; ++w)
    if (tops[w] > top || (tops[w] == top && ats[w] < at)) { top = tops[w]; at = ats[w]; }
  double s = 0.0;
  if (!greedy && at != INT_MAX) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += weight(x[j][e], top, inv);
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) a.part[(int64_t)r * a.chunks + c] = Part{s, top, at};
}

// A row's maximum, the first index of it, and its sum, by one wave.
__device__ __forceinline__ Part row_total(const Part* part, int chunks, double inv) {
  const int lane = threadIdx.x & 63;
  float top = -INFINITY;
  int at = INT_MAX;
  for (int c = lane; c < chunks; c += 64)
    if (part[c].top > top) { top = part[c].top; at = part[c].at; }
  for (int o = 32; o > 0; o >>= 1) {
    const float ot = __shfl_xor(top, o, 64);
    const int oa = __shfl_xor(at, o, 64);
    if (ot > top || (ot == top && oa < at)) { top = ot; at = oa; }
  }
  double s = 0.0;
  for (int c = lane; c < chunks; c += 64) s += part[c].sum * weight(part[c].top, top, inv);
  return Part{wave_sum_f64(s), top, at};
}

// The decision (by every workgroup of a sequence for itself: a few partials from L2
// cost less than one more kernel), and the chunk's share of what the next token is
// drawn from.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_decide_kernel(Verify<T> a) {
  __shared__ double sh[kThreads / 64];
  __shared__ int first;
  const int b = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks;
  const int wave = threadIdx.x >> 6;
  const int n = a.drafts(b);
  bool greedy;
  const double inv = a.inverse(b, &greedy);
  if (threadIdx.x == 0) first = n;
  __syncthreads();
  for (int i = wave; i < n; i += kThreads / 64) {
    const Part p = row_total(a.target_part(b, i), a.chunks, inv);
    const int x = a.tokens[(int64_t)b * a.g + i];
    const bool in = x >= 0 && x < a.vocab;
    bool keep;
    if (greedy) {
      keep = in && x == p.at;
    } else {
      double qx = a.draft ? 0.0 : 1.0;
      if (a.draft && in) {
        const Part q = row_total(a.draft_part(b, i), a.chunks, inv);
        if (q.sum > 0.0) qx = weight(ld(a.draft_row(b, i) + x), q.top, inv) / q.sum;
      }
      const double px =
          in && p.sum > 0.0 ? weight(ld(a.target_row(b, i) + x), p.top, inv) / p.sum : 0.0;
      keep = (double)a.u[(int64_t)b * (a.g + 1) + i] * qx < px;
    }
    if (!keep && (threadIdx.x & 63) == 0) atomicMin(&first, i);
  }
  __syncthreads();
  const int kept = first;
  const Part p = row_total(a.target_part(b, kept), a.chunks, inv);
  Part q{0.0, 0.0f, 0};
  Pick k{};
  k.kept = kept;
  k.at = p.at;
  k.mode = greedy ? kPickGreedy : kept == n ? kPickRow : a.draft ? kPickRest : kPickOthers;
  if (k.mode == kPickRest) {
    q = row_total(a.draft_part(b, kept), a.chunks, inv);
    if (q.sum <= 0.0) k.mode = kPickRow;
  }
  if (k.mode == kPickOthers) k.gone = a.tokens[(int64_t)b * a.g + kept];
  k.p_total = p.sum;
  k.p_top = p.top;
  k.q_total = q.sum;
  k.q_top = q.top;
  if (c == 0 && threadIdx.x == 0) a.pick[b] = k;
  if (k.mode == kPickGreedy || !(p.sum > 0.0)) return;
  const T* row = a.target_row(b, kept);
  const Part own = a.target_part(b, kept)[c];
  double s = own.sum * weight(own.top, p.top, inv);
  const int lo = c * kChunk - (k.mode == kPickRest ? 0 : lead_of(row));
  if (k.mode == kPickRest || (k.mode == kPickOthers && k.gone >= lo && k.gone < lo + kChunk)) {
    const T* other = k.mode == kPickRest ? a.draft_row(b, kept) : row;
    s = 0.0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int v = lo + j * kThreads + (int)threadIdx.x;
      if (v < 0 || v >= a.vocab) continue;
      const double w = weight(ld(row + v), p.top, inv);
      if (k.mode == kPickRest)
        s += fmax(w / p.sum - weight(ld(other + v), q.top, inv) / q.sum, 0.0);
      else
        s += v == k.gone ? 0.0 : w;
    }
    s = block_sum(s, sh);
  }
  if (threadIdx.x == 0) a.rest[(int64_t)b * a.chunks + c] = s;
}

// The next token of a sequence: the first index whose running sum passes u times the
// whole.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(Verify<T> a) {
  __shared__ double sh[kThreads / 64];
  __shared__ int found, last;
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Pick k = a.pick[b];
  bool greedy;
  const double inv = a.inverse(b, &greedy);
  int next = -1;
  if (greedy) {
    if (k.at != INT_MAX) next = k.at;
  } else if (k.p_total > 0.0) {
    const T* row = a.target_row(b, k.kept);
    const Part* part = a.target_part(b, k.kept);
    // every wave for itself, 64 chunks at a time
    auto mass = [&](int c) {
      if (c >= a.chunks) return 0.0;
      return k.mode == kPickRow ? part[c].sum * weight(part[c].top, k.p_top, inv)
                                : a.rest[(int64_t)b * a.chunks + c];
    };
    auto whole = [&]() {
      double s = 0.0;
      for (int c = lane; c < a.chunks; c += 64) s += mass(c);
      return wave_sum_f64(s);
    };
    double total = whole();
    if (k.mode != kPickRow && !(total > 0.0)) {   // p is q: nothing is left of it
      k.mode = kPickRow;
      total = whole();
    }
    const double r = (double)a.u[(int64_t)b * (a.g + 1) + a.g];
    const double aim = r > 0.0 ? r * total : 0.0;
    double before = 0.0;        // the sum of the chunks before `chunk`
    int chunk = -1;
    double run = 0.0;
    for (int c0 = 0; c0 < a.chunks; c0 += 64) {
      const double m = mass(c0 + lane);
      double s = m;
      for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(s, o, 64);
        if (lane >= o) s += t;
      }
      // the chunk that passes the aim, else the last one that holds something
      const uint64_t over = __ballot(m > 0.0 && run + s > aim);
      const uint64_t some = __ballot(m > 0.0);
      const int hit = over ? __ffsll((unsigned long long)over) - 1
                           : some ? 63 - __clzll((long long)some) : -1;
      if (hit >= 0) {
        chunk = c0 + hit;
        before = run + __shfl(s - m, hit, 64);
      }
      if (over) break;
      run += __shfl(s, 63, 64);
    }
    if (threadIdx.x == 0) {
      found = INT_MAX;
      last = -1;
    }
    __syncthreads();
    if (chunk >= 0) {
      const int lo = chunk * kChunk - (k.mode == kPickRest ? 0 : lead_of(row)) +
                     (int)threadIdx.x * kPer;
      const T* other = k.mode == kPickRest ? a.draft_row(b, k.kept) : row;
      double w[kPer], s = 0.0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int v = lo + e;
        w[e] = 0.0;
        if (v >= 0 && v < a.vocab) {
          w[e] = weight(ld(row + v), k.p_top, inv);
          if (k.mode == kPickRest)
            w[e] = fmax(w[e] / k.p_total - weight(ld(other + v), k.q_top, inv) / k.q_total, 0.0);
          else if (k.mode == kPickOthers && v == k.gone)
            w[e] = 0.0;
        }
        s += w[e];
      }
      double scan = s;
      for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(scan, o, 64);
        if (lane >= o) scan += t;
      }
      if (lane == 63) sh[wave] = scan;
      __syncthreads();
      double at = before + (scan - s);
      for (int v = 0; v < wave; ++v) at += sh[v];
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        at += w[e];
        if (w[e] > 0.0) {
          if (at > aim) atomicMin(&found, lo + e);
          atomicMax(&last, lo + e);
        }
      }
    }
    __syncthreads();
    next = found != INT_MAX ? found : last;
  }
  for (int i = threadIdx.x; i <= a.g; i += kThreads)
    a.out[(int64_t)b * (a.g + 1) + i] =
        i < k.kept ? a.tokens[(int64_t)b * a.g + i] : i == k.kept ? next : -1;
  if (threadIdx.x == 0) a.kept[b] = k.kept;
}

int chunks_of(int vocab) { return ceil_div((long)vocab + 7, kChunk); }   // 7: the largest lead
struct VerifyWs {
  size_t part, rest, pick, total;
};
VerifyWs verify_ws(int64_t n_seq, int64_t g, int vocab) {
  auto align = [](size_t x) { return (x + 255) / 256 * 256; };
  const int64_t c = chunks_of(vocab);
  VerifyWs w{};
  w.part = 0;
  w.rest = align((size_t)(n_seq * (2 * g + 1) * c) * sizeof(Part));
  w.pick = w.rest + align((size_t)(n_seq * c) * sizeof(double));
  w.total = w.pick + align((size_t)n_seq * sizeof(Pick));
  return w;
}

template <typename T>
adept_status verify_launch(Verify<T> a, void* workspace, hipStream_t s) {
  const VerifyWs w = verify_ws(a.n_seq, a.g, a.vocab);
  a.chunks = chunks_of(a.vocab);
  a.part = (Part*)((char*)workspace + w.part);
  a.rest = (double*)((char*)workspace + w.rest);
  a.pick = (Pick*)((char*)workspace + w.pick);
  const int rows = a.n_seq * (a.g + 1) + (a.draft ? a.n_seq * a.g : 0);
  ADEPT_LAUNCH(verify_rows_kernel<T>, dim3((unsigned)rows * a.chunks), dim3(kThreads), 0, s, a);
  ADEPT_CHECK_LAUNCH("verify_rows");
  ADEPT_LAUNCH(verify_decide_kernel<T>, dim3((unsigned)a.n_seq * a.chunks), dim3(kThreads), 0, s, a);
  ADEPT_CHECK_LAUNCH("verify_decide");
  ADEPT_LAUNCH(verify_pick_kernel<T>, dim3(a.n_seq), dim3(kThreads), 0, s, a);
  return launch_status("verify_pick");
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
