// Attention of new tokens over a paged cache (adept_paged_attend).
//
// Tiles (bf16 queries, head_dim 64 / 128): the (entry, query head) pairs that
// read one K/V head of one sequence are the columns of a matrix; a plan kernel
// cuts each sequence's columns into tiles of 128.  A workgroup takes one (tile,
// K/V head) and, where there are too few of those to fill the card, a part of
// the keys, which a second kernel joins.
//
// Walk (f32, other widths): one wave per (entry, head) takes the keys one after
// another: lane l holds the dims l, l + 64, ... of q and of the running output,
// a score is a sum over the wave.  A key that is not seen is skipped, whatever
// it holds.
//
// A key that some columns of a tile see and others do not (a later token of the
// chunk) has weight 0 in the matrix product of the others, which is no 0 where
// its V is infinite or NaN.  A tile whose result is not finite is therefore
// computed again by the walk, column by column.
#include <algorithm>

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

// The walk of one wave over the keys t0 .. t1-1 of a sequence for one query
// (R dims per lane): running maximum m (in the exp2 domain), sum l and output o.
template <int R>
struct Walk {
  float m, l, o[R];
};
template <typename T, typename TC, int R>
__device__ __forceinline__ Walk<R> walk_keys(const T* __restrict__ q, int hd, float scale_log2,
                                             const PagedView& c, const int32_t* __restrict__ pages,
                                             int hk, int t0, int t1) {
  const int lane = threadIdx.x & 63;
  float qv[R];
  Walk<R> w{-INFINITY, 0.0f, {}};
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int d = lane + 64 * i;
    qv[i] = d < hd ? ld(q + d) * scale_log2 : 0.0f;
    w.o[i] = 0.0f;
  }
  for (int t = t0; t < t1; ++t) {
    const int s = c.slot(pages, t);
    if (s < 0) continue;
    const int64_t row = (int64_t)s * c.n_kv_heads + hk;
    float x = 0.0f, v[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int d = lane + 64 * i;
      v[i] = 0.0f;
      if (d >= hd) continue;
      x = fmaf(qv[i], cache_value<TC>(c.k, c.k_scale, row, hd, d), x);
      v[i] = cache_value<TC>(c.v, c.v_scale, row, hd, d);
    }
    x = wave_sum_f32(x);
    if (x == -INFINITY) continue;      // no weight
    const float mn = fmaxf(w.m, x);
    const float a = exp2f(w.m - mn), p = exp2f(x - mn);
    w.m = mn;
    w.l = fmaf(w.l, a, p);
#pragma unroll
    for (int i = 0; i < R; ++i) w.o[i] = fmaf(p, v[i], w.o[i] * a);
  }
  return w;
}

template <typename T, int R>
__device__ __forceinline__ void walk_store(const Walk<R>& w, int hd, T* __restrict__ out) {
  const float inv = w.l == 0.0f ? 0.0f : 1.0f / w.l;   // no key: zeros
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int d = (threadIdx.x & 63) + 64 * i;
    if (d < hd) st(out + d, w.o[i] * inv);
  }
}

template <typename T, typename TC>
__global__ __launch_bounds__(256) void paged_attend_walk_kernel(int H, int hd, float scale_log2,
                                                                const T* __restrict__ q, Entries e,
                                                                PagedView c, T* __restrict__ out) {
  const int k = blockIdx.x, h = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (k >= min(*e.n_active, e.max_active) || h >= H) return;
  int b;
  const int n = entry_limit(e, c, e.rows[k], &b);
  const int64_t at = ((int64_t)k * H + h) * hd;
  walk_store(walk_keys<T, TC, 4>(q + at, hd, scale_log2, c, c.table + (int64_t)b * c.max_pages,
                                 h / (H / c.n_kv_heads), 0, n),
             hd, out + at);
}

// ---------------------------------------------------------------------------
// plan of the tiles
// ---------------------------------------------------------------------------
constexpr int TC_ = 128;       // columns of a tile
constexpr int kPlanThreads = 1024;

// Columns of one sequence's entries (a stretch of the list from entry `first`
// on, G columns each): columns col .. col + cols - 1, cols <= TC_.
struct Tile {
  int first, col, cols, seq;
};

// Segments: stretches of entries of one sequence.  Each pass takes 8 entries of
// every thread, all loads of the pass in flight together, and ranks the starts
// by wave ballots; then a scan over the segments' tile counts.  starts:
// [max_active + 1].
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(Entries e, int G,
                                                                  int32_t* __restrict__ starts,
                                                                  Tile* __restrict__ tiles,
                                                                  int32_t* __restrict__ n_tiles) {
  constexpr int U = 8, W = kPlanThreads / 64;
  __shared__ int cnt[U * W], base_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(*e.n_active, e.max_active);
  if (tid == 0) base_s = 0;
  for (int k0 = 0; k0 < n; k0 += U * kPlanThreads) {
    int at[U], before[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * kPlanThreads + tid;
      at[u] = k < n ? e.rows[k] : -1;
      before[u] = k > 0 && k < n ? e.rows[k - 1] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      at[u] = at[u] >= 0 ? e.seq[at[u]] : 0;
      before[u] = before[u] >= 0 ? e.seq[before[u]] : at[u] + 1;
    }
    uint64_t m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      m[u] = __ballot(k0 + u * kPlanThreads + tid < n && at[u] != before[u]);
      if (lane == 0) cnt[u * W + wave] = __popcll(m[u]);
    }
    __syncthreads();
    if (wave == 0) {               // exclusive ranks of the U * W = 128 counts
      const int a = cnt[2 * lane], b = cnt[2 * lane + 1];
      int x = a + b;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
      }
      const int base = base_s + x - a - b;
      cnt[2 * lane] = base;
      cnt[2 * lane + 1] = base + a;
      if (lane == 63) base_s += x;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if ((m[u] >> lane) & 1)
        starts[cnt[u * W + wave] + __popcll(m[u] & ((1ull << lane) - 1))] =
            k0 + u * kPlanThreads + tid;
    __syncthreads();
  }
  const int ns = n > 0 ? base_s : 0;
  if (tid == 0) starts[ns] = n;
  __syncthreads();                 // starts are this workgroup's own writes
  if (wave != 0) return;
  int acc = 0;
  for (int i0 = 0; i0 < ns; i0 += 64) {
    const int i = i0 + lane;
    const int first = i < ns ? starts[i] : 0;
    const int64_t cols = i < ns ? (int64_t)(starts[i + 1] - first) * G : 0;
    const int nt = (int)((cols + TC_ - 1) / TC_);
    int x = nt;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    const int seq = i < ns ? e.seq[e.rows[first]] : 0;
    for (int t = 0; t < nt; ++t)
      tiles[acc + x - nt + t] =
          Tile{first, t * TC_, (int)min((int64_t)TC_, cols - (int64_t)t * TC_), seq};
    acc += __shfl(x, 63, 64);
  }
  if (lane == 0) *n_tiles = acc;
}

// ---------------------------------------------------------------------------
// tiles
// ---------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
constexpr float kLazy = 8.0f;   // log2 headroom of the reference maximum
constexpr int KB = 64;          // keys of a block
constexpr int kTileThreads = 256;

// What takes the place of the K and V rows of keys that no column sees.
__device__ const uint4 kZeroRow[16] = {};

// max(a, b, c) without quieting the matrix products' results first (fmaxf
// would: one more instruction a value)
__device__ __forceinline__ float max3_raw(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// max over lanes l and l ^ 32
__device__ __forceinline__ float max_halves(float m) {
  const uint32_t u = __float_as_uint(m);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return max3_raw(m, __uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ bool finite(float x) {
  return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u;
}

// Column j of a tile: its entry and query head.
__device__ __forceinline__ void column_of(const Tile& t, int j, int G, int hk, int* k, int* h) {
  const int c = t.col + j;
  *k = t.first + c / G;
  *h = hk * G + c % G;
}

// One workgroup per (tile, K/V head, part of the keys).  Wave w holds columns
// 32 w .. 32 w + 31.  Scores come transposed, S^T = K Q^T (32 keys x 32 columns,
// v_mfma_f32_32x32x16_bf16): lanes l and l + 32 hold one column's scores, the
// first the keys 8 i + 0 .. 3, the second 8 i + 4 .. 7, so a column's maximum
// takes one lane swap, and the weights already lie as the B operand of
// O^T += V^T P^T wants them, if V^T is read in the same order of keys.
//
// K and V come in blocks of 64 keys, bf16 in LDS in two stages, block kb + 1
// on its way while block kb is computed.  A bf16 cache is copied there by
// direct loads; an 8-bit one goes through registers, where its codes become
// bf16 with their scale in the conversion itself (exactly).  The slot of key
// t0 + lane is found by every wave one block ahead; its ballot is the mask of
// the keys that are there, and the others' rows are read from a row of zeros,
// so that they add nothing whatever the cache holds.
//
// Chunk c (16 bytes) of row r lies at c ^ fk(r) in K, c ^ fv(r) in V: the K
// reads (32 rows, two chunks) and the transposing V reads (4 rows, 4 chunks in
// each half) then fall on distinct banks.
template <int HD, bool FP8>
__global__ __launch_bounds__(kTileThreads, 2) void paged_tile_kernel(
    int H, float scale_log2, const bf16* __restrict__ q, Entries e, PagedView c,
    const Tile* __restrict__ tiles, const int32_t* __restrict__ n_tiles, int max_tiles, int parts,
    bf16* __restrict__ out, float* __restrict__ part) {
  constexpr int DS = HD / 16;               // 16-dim steps of S
  constexpr int DB = HD / 32;               // 32-dim blocks of O^T
  constexpr int ROWB = HD * 2;              // bytes of a row in LDS
  constexpr int NCH = ROWB / 16;            // its 16-byte chunks
  constexpr int RPI = 1024 / ROWB;          // rows of one direct load of a wave
  constexpr int DPW = KB / RPI / 4;         // direct loads of a wave and operand
  constexpr int BLK = KB * ROWB;
  // 8-bit cache: 16-byte pieces of a row, and how many of a block a thread takes
  constexpr int PCH = HD / 16, PPT = KB * PCH / kTileThreads;
  __shared__ __attribute__((aligned(1024))) char sKV[2][2][BLK];

  const int G = H / c.n_kv_heads;
  const int nt = *n_tiles;
  // Work items head by head.  The hardware deals workgroups round-robin to the
  // 8 XCDs: with 8 K/V heads or more each XCD takes a run of items, so that the
  // tiles in flight on it share a few heads' K/V in its L2; with fewer heads the
  // items are dealt as they come, which keeps the XCDs evenly loaded.
  const int total = max_tiles * c.n_kv_heads * parts;
  int item = blockIdx.x;
  if (c.n_kv_heads >= 8) {
    const int per = (total + 7) >> 3;
    item = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per) return;
  }
  if (item >= total) return;
  const int p = item % parts, ti0 = item / parts % max_tiles, hk = item / parts / max_tiles;
  // a list whose sequences are scattered can hold more tiles than the host
  // counted on: then each workgroup takes several, with all of their keys
  const bool whole = parts == 1 || nt > max_tiles;
  if (whole && p > 0) return;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, c32 = lane & 31;
  auto fk = [](int r) { return HD == 128 ? (r & 15) : ((r >> 1) & 7); };
  auto fv = [](int r) { return HD == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); };

  for (int ti = ti0; ti < nt; ti += max_tiles) {
    const Tile tile = tiles[nt - 1 - ti];   // of a prompt, the latest (longest) first
    const int32_t* pages = c.table + (int64_t)tile.seq * c.max_pages;
    // keys that some column sees, this wave's columns, and this lane's column
    int tend = 0, wend = 0, wfull = INT_MAX, qlim = 0;
    for (int j = lane; j < tile.cols; j += 64) {
      int k, h, b;
      column_of(tile, j, G, hk, &k, &h);
      tend = max(tend, entry_limit(e, c, e.rows[k], &b));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) tend = max(tend, __shfl_xor(tend, o, 64));
    tend = __builtin_amdgcn_readfirstlane(tend);
    const int j = wave * 32 + c32;
    const bool valid = j < tile.cols;
    int qk, qh;
    column_of(tile, valid ? j : 0, G, hk, &qk, &qh);
    const int64_t qat = ((int64_t)qk * H + qh) * HD;
    if (valid) {
      int b;
      qlim = entry_limit(e, c, e.rows[qk], &b);
    }
    wend = qlim;
    wfull = valid ? qlim : INT_MAX;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      wend = max(wend, __shfl_xor(wend, o, 64));
      wfull = min(wfull, __shfl_xor(wfull, o, 64));
    }
    wend = __builtin_amdgcn_readfirstlane(wend);
    wfull = __builtin_amdgcn_readfirstlane(wfull);   // keys below it: every column sees them
    // this part's keys
    int tb = 0, te = tend;
    if (!whole) {
      const int per = ((tend + KB - 1) / KB + parts - 1) / parts * KB;
      tb = min(p * per, tend);
      te = min(tb + per, tend);
    }
    const int nkb = (te - tb + KB - 1) / KB;

    bf16x8_t qf[DS];
#pragma unroll
    for (int s = 0; s < DS; ++s)
      qf[s] = __builtin_bit_cast(bf16x8_t,
                                 *reinterpret_cast<const uint4*>(q + qat + s * 16 + hh * 8));
    f32x16_t o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[i][v] = 0.0f;
    float m_ref = -INFINITY, l_run = 0.0f;

    // slots of a block's keys, one per lane
    auto slots_of = [&](int kb) {
      const int t = tb + kb * KB + lane;
      return t < te ? c.slot(pages, t) : -1;
    };
    const int64_t rowc = (int64_t)c.n_kv_heads * HD;    // elements of a slot
    // bf16: direct loads
    auto issue = [&](int u, int sl) {
#pragma unroll
      for (int jj = 0; jj < DPW; ++jj) {
        const int qd = wave * DPW + jj;
        const int r = qd * RPI + lane / NCH;
        const int s = __shfl(sl, r, 64);
        const int64_t at = s * rowc + hk * HD;
#pragma unroll
        for (int op = 0; op < 2; ++op) {
          const int ch = (lane % NCH) ^ (op ? fv(r) : fk(r));
          const char* src = (const char*)((const bf16*)(op ? c.v : c.k) + at) + ch * 16;
          if (s < 0) src = (const char*)kZeroRow + ch * 16;
          __builtin_amdgcn_global_load_lds(
              (__attribute__((address_space(1))) void*)src,
              (__attribute__((address_space(3))) void*)(&sKV[u][op][qd * 1024]), 16, 0, 0);
        }
      }
    };
    // 8-bit: codes and scales to registers, then as bf16 to LDS
    uint4 code[2][PPT];
    float csc[2][PPT];
    auto fetch = [&](int sl) {
#pragma unroll
      for (int i = 0; i < PPT; ++i) {
        const int pc = i * kTileThreads + tid, r = pc / PCH;
        const int s = __shfl(sl, r, 64);
#pragma unroll
        for (int op = 0; op < 2; ++op) {
          code[op][i] = make_uint4(0, 0, 0, 0);
          csc[op][i] = 1.0f;
          if (s >= 0) {
            const uint8_t* src = (const uint8_t*)(op ? c.v : c.k) + s * rowc + hk * HD;
            code[op][i] = *reinterpret_cast<const uint4*>(src + pc % PCH * 16);
            csc[op][i] = scale_of((op ? c.v_scale : c.k_scale)[(int64_t)s * c.n_kv_heads + hk]);
          }
        }
      }
    };
    auto put = [&](int u) {
#pragma unroll
      for (int i = 0; i < PPT; ++i) {
        const int pc = i * kTileThreads + tid, r = pc / PCH;
#pragma unroll
        for (int op = 0; op < 2; ++op) {
          const uint32_t w[4] = {code[op][i].x, code[op][i].y, code[op][i].z, code[op][i].w};
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint4 x = make_uint4(fp8x2_to_bf16x2<false>(w[2 * half], csc[op][i]),
                                       fp8x2_to_bf16x2<true>(w[2 * half], csc[op][i]),
                                       fp8x2_to_bf16x2<false>(w[2 * half + 1], csc[op][i]),
                                       fp8x2_to_bf16x2<true>(w[2 * half + 1], csc[op][i]));
            const int ch = (pc % PCH * 2 + half) ^ (op ? fv(r) : fk(r));
            *reinterpret_cast<uint4*>(&sKV[u][op][r * ROWB + ch * 16]) = x;
          }
        }
      }
    };

    uint64_t there = 0;
    int sl = -1;
    if (nkb > 0) {
      sl = slots_of(0);
      there = __ballot(sl >= 0);
      if constexpr (FP8) {
        fetch(sl);
        put(0);
      } else {
        issue(0, sl);
      }
      sl = nkb > 1 ? slots_of(1) : -1;
    }
    __syncthreads();
    for (int kb = 0; kb < nkb; ++kb) {
      const int u = kb & 1, t0 = tb + kb * KB;
      const uint64_t mask = there;
      // the other stage was last read in block kb - 1
      if (kb + 1 < nkb) {
        there = __ballot(sl >= 0);
        if constexpr (FP8) fetch(sl); else issue(u ^ 1, sl);
        sl = kb + 2 < nkb ? slots_of(kb + 2) : -1;
      }
      if (t0 < wend) {
        const char* cK = sKV[u][0];
        const char* cV = sKV[u][1];
        // S^T = K Q^T
        __builtin_amdgcn_s_setprio(1);
        f32x16_t s[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
          for (int v = 0; v < 16; ++v) s[kt][v] = 0.0f;
          const int r = kt * 32 + c32;
#pragma unroll
          for (int ds = 0; ds < DS; ++ds) {
            const bf16x8_t a = *reinterpret_cast<const bf16x8_t*>(
                cK + r * ROWB + ((2 * ds + hh) ^ fk(r)) * 16);
            s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[ds], s[kt], 0, 0, 0);
          }
        }
        __builtin_amdgcn_s_setprio(0);
        // keys that are not there, or past a column's end
        if (t0 + KB > wfull || mask != ~0ull) {
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const int kl = kt * 32 + 8 * (v >> 2) + 4 * hh + (v & 3);
              const bool keep = t0 + kl < qlim && ((mask >> kl) & 1);
              s[kt][v] = keep ? s[kt][v] : -INFINITY;
            }
        }
        // the block's maximum of the column; the reference maximum moves (and o
        // is rescaled) only where a block exceeds it by more than 2^kLazy
        float mb = max3_raw(s[0][0], s[0][1], s[0][2]);
#pragma unroll
        for (int v = 3; v < 15; v += 2) mb = max3_raw(mb, s[0][v], s[0][v + 1]);
        mb = max3_raw(mb, s[0][15], s[1][0]);
#pragma unroll
        for (int v = 1; v < 15; v += 2) mb = max3_raw(mb, s[1][v], s[1][v + 1]);
        mb = max_halves(max3_raw(mb, s[1][15], mb)) * scale_log2;
        if (__any(mb > m_ref + kLazy)) {
          const float mn = fmaxf(m_ref, mb);
          const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_ref - mn);
          m_ref = mn;
          l_run *= alpha;
#pragma unroll
          for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[i][v] *= alpha;
        }
        // weights, rounded to bf16 (the sum takes the rounded ones, as the
        // product does), as the B operand: 16 keys a step
        bf16x8_t pb[4];
        const float msub = m_ref == -INFINITY ? 0.0f : m_ref;
        constexpr bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t w[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float a = s[i >> 1][8 * (i & 1) + 2 * x], b = s[i >> 1][8 * (i & 1) + 2 * x + 1];
            w[x] = pack_bf16x2(__builtin_amdgcn_exp2f(fmaf(a, scale_log2, -msub)),
                               __builtin_amdgcn_exp2f(fmaf(b, scale_log2, -msub)));
            l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[x]), ones,
                                                    l_run, false);
          }
          pb[i] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
        }
        // O^T += V^T P^T: in each 16-lane group source lane L reads 4 dims of
        // key k0 + L/4 and lane i receives dim n0 + i of keys k0 .. k0 + 3
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s16x4 half[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int r = 16 * i + 8 * x + 4 * hh + ((lane & 15) >> 2);
              const int ch = db * 4 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
              half[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (lds_s16x4*)(cV + r * ROWB + ((ch ^ fv(r)) * 16) + 8 * (lane & 1)));
            }
            const bf16x8_t a = __builtin_bit_cast(
                bf16x8_t, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[i], o[db], 0, 0, 0);
          }
        __builtin_amdgcn_s_setprio(0);
      }
      if constexpr (FP8) {
        if (kb + 1 < nkb) put(u ^ 1);
      }
      __syncthreads();   // block kb + 1 landed, stage u is free
    }

    const float l = l_run + __shfl_xor(l_run, 32, 64);
    bool ok = finite(l);
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) ok &= finite(o[i][v]);
    const uint64_t bad = __ballot(valid && !ok);
    const uint32_t redo = (uint32_t)bad | (uint32_t)(bad >> 32);   // by column
    float* pp = nullptr;     // this column's partial result: m, l, then the dims
    if (!whole) pp = part + (((int64_t)(nt - 1 - ti) * c.n_kv_heads + hk) * parts + p) * TC_ * (HD + 2);
    if (valid && !((redo >> c32) & 1)) {
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
          const int d = db * 32 + 2 * v + 4 * hh;
          if (whole) {
            *reinterpret_cast<uint2*>(out + qat + d) =
                make_uint2(pack_bf16x2(o[db][v] * inv, o[db][v + 1] * inv),
                           pack_bf16x2(o[db][v + 2] * inv, o[db][v + 3] * inv));
          } else {
            *reinterpret_cast<float4*>(pp + TC_ * 2 + j * HD + d) =
                make_float4(o[db][v], o[db][v + 1], o[db][v + 2], o[db][v + 3]);
          }
        }
      if (!whole && hh == 0) *reinterpret_cast<float2*>(pp + 2 * j) = make_float2(m_ref, l);
    }
    for (uint32_t left = redo; left; left &= left - 1) {
      const int x = __ffs(left) - 1, jj = wave * 32 + x;
      int k, h;
      column_of(tile, jj, G, hk, &k, &h);
      const int lim = min(__shfl(qlim, x, 64), te);
      const int64_t at = ((int64_t)k * H + h) * HD;
      const auto w = walk_keys<bf16, typename std::conditional<FP8, uint8_t, bf16>::type, HD / 64>(
          q + at, HD, scale_log2, c, pages, hk, tb, lim);
      if (whole) {
        walk_store(w, HD, out + at);
      } else {
        for (int i = 0; i < HD / 64; ++i) pp[TC_ * 2 + jj * HD + lane + 64 * i] = w.o[i];
        if (lane == 0) *reinterpret_cast<float2*>(pp + 2 * jj) = make_float2(w.m, w.l);
      }
    }
    __syncthreads();     // the next tile's loads overwrite the stages
  }
}

// Joins the parts of each (tile, K/V head): a thread takes four dims of a column.
template <int HD>
__global__ __launch_bounds__(256) void paged_tile_join_kernel(
    int H, Entries e, int n_kv_heads, const Tile* __restrict__ tiles,
    const int32_t* __restrict__ n_tiles, int max_tiles, int parts, const float* __restrict__ part,
    bf16* __restrict__ out) {
  constexpr int CPB = 256 / (HD / 4);      // columns of a workgroup
  const int ti = blockIdx.x, hk = blockIdx.y, nt = *n_tiles;
  if (ti >= nt || nt > max_tiles) return;
  const Tile tile = tiles[ti];
  const int G = H / n_kv_heads;
  const int j = blockIdx.z * CPB + threadIdx.x / (HD / 4), d = threadIdx.x % (HD / 4) * 4;
  if (j >= tile.cols) return;
  const float* pp = part + ((int64_t)ti * n_kv_heads + hk) * parts * TC_ * (HD + 2);
  float m = -INFINITY;
  for (int p = 0; p < parts; ++p) m = fmaxf(m, pp[(int64_t)p * TC_ * (HD + 2) + 2 * j]);
  float l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = 0; p < parts; ++p) {
    const float* x = pp + (int64_t)p * TC_ * (HD + 2);
    const float2 ml = *reinterpret_cast<const float2*>(x + 2 * j);
    const float4 v = *reinterpret_cast<const float4*>(x + TC_ * 2 + j * HD + d);
    if (ml.x == -INFINITY && ml.y == 0.0f) continue;    // a part without keys
    const float w = __builtin_amdgcn_exp2f(ml.x - m);
    l = fmaf(w, ml.y, l);
    o[0] = fmaf(w, v.x, o[0]);
    o[1] = fmaf(w, v.y, o[1]);
    o[2] = fmaf(w, v.z, o[2]);
    o[3] = fmaf(w, v.w, o[3]);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  int k, h;
  column_of(tile, j, G, hk, &k, &h);
  *reinterpret_cast<uint2*>(out + ((int64_t)k * H + h) * HD + d) =
      make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
}

// Tiles that the host counts on, and the parts of the keys with which they make
// about two workgroups a CU (a part keeps at least 256 of the keys there may be).
struct TileShape {
  int max_tiles, cap_tiles, parts;
  size_t off_tiles, off_starts, off_part, bytes;
};
TileShape tile_shape(const adept_paged_kv& kv, int n_heads, int max_active, int n_seq,
                     int max_pages) {
  const int64_t G = n_heads / kv.n_kv_heads, keys = (int64_t)max_pages * kv.page_size;
  TileShape t{};
  const int64_t full = max_active * G / TC_;
  t.max_tiles = (int)(full + std::min(n_seq, max_active));
  t.cap_tiles = (int)(full + max_active);
  const int64_t base = (int64_t)t.max_tiles * kv.n_kv_heads;
  t.parts = (int)std::max<int64_t>(1, std::min<int64_t>({512 / std::max<int64_t>(base, 1),
                                                         (keys + 255) / 256, 32}));
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  t.off_tiles = 256;
  t.off_starts = t.off_tiles + up((size_t)t.cap_tiles * sizeof(Tile));
  t.off_part = t.off_starts + up(((size_t)max_active + 1) * sizeof(int32_t));
  t.bytes = t.off_part;
  if (t.parts > 1) t.bytes += (size_t)base * t.parts * TC_ * (kv.head_dim + 2) * sizeof(float);
  return t;
}

bool tiles_fit(adept_dtype dt, const adept_paged_kv& kv) {
  return dt == ADEPT_BF16 && (kv.head_dim == 64 || kv.head_dim == 128);
}

}  // namespace
}  // namespace adept

using namespace adept;

extern "C" size_t adept_paged_attend_workspace_bytes(const adept_paged_kv* kv, int n_heads,
                                                     int max_active, int n_seq, int max_pages) {
  if (!kv || kv->n_kv_heads <= 0 || n_heads < kv->n_kv_heads || max_active < 0 || n_seq <= 0 ||
      max_pages <= 0)
    return 256;
  return tile_shape(*kv, n_heads, max_active, n_seq, max_pages).bytes;
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
  const bool fp8 = kv->dtype == ADEPT_KV_FP8;
  if (tiles_fit(dt, *kv)) {
    const TileShape ts = tile_shape(*kv, n_heads, max_active, n_seq, max_pages);
    char* w = (char*)workspace;
    int32_t* n_tiles = (int32_t*)w;
    Tile* tiles = (Tile*)(w + ts.off_tiles);
    float* part = (float*)(w + ts.off_part);
    const int64_t items = (int64_t)ts.max_tiles * kv->n_kv_heads * ts.parts;
    ADEPT_REQUIRE(items <= 1 << 23, "paged_attend: too many entries");
    ADEPT_LAUNCH(paged_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, e, n_heads / kv->n_kv_heads,
                 (int32_t*)(w + ts.off_starts), tiles, n_tiles);
    ADEPT_CHECK_LAUNCH("paged_plan");
#define ADEPT_TILE(HD, FP8)                                                                      \
  ADEPT_LAUNCH((paged_tile_kernel<HD, FP8>), dim3((unsigned)((items + 7) / 8 * 8)),              \
               dim3(kTileThreads), 0, s, n_heads, sl, (const bf16*)q, e, c, tiles, n_tiles,      \
               ts.max_tiles, ts.parts, (bf16*)out, part)
    if (hd == 128) {
      if (fp8) ADEPT_TILE(128, true); else ADEPT_TILE(128, false);
    } else {
      if (fp8) ADEPT_TILE(64, true); else ADEPT_TILE(64, false);
    }
#undef ADEPT_TILE
    ADEPT_CHECK_LAUNCH("paged_tile");
    if (ts.parts > 1) {
      const dim3 jg(ts.max_tiles, kv->n_kv_heads, TC_ * hd / 1024);
      if (hd == 128)
        ADEPT_LAUNCH(paged_tile_join_kernel<128>, jg, dim3(256), 0, s, n_heads, e, kv->n_kv_heads,
                     tiles, n_tiles, ts.max_tiles, ts.parts, part, (bf16*)out);
      else
        ADEPT_LAUNCH(paged_tile_join_kernel<64>, jg, dim3(256), 0, s, n_heads, e, kv->n_kv_heads,
                     tiles, n_tiles, ts.max_tiles, ts.parts, part, (bf16*)out);
    }
    return launch_status("paged_attend");
  }
  const dim3 grid(max_active, ceil_div(n_heads, 4));
#define ADEPT_WALK(T, TC)                                                                       \
  ADEPT_LAUNCH((paged_attend_walk_kernel<T, TC>), grid, dim3(256), 0, s, n_heads, hd, sl,       \
               (const T*)q, e, c, (T*)out)
  if (dt == ADEPT_F32) {
    if (fp8) ADEPT_WALK(float, uint8_t); else ADEPT_WALK(float, float);
  } else {
    if (fp8) ADEPT_WALK(bf16, uint8_t); else ADEPT_WALK(bf16, bf16);
  }
#undef ADEPT_WALK
  return launch_status("paged_attend");
}
