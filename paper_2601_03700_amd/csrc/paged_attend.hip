// Attention of new tokens over a paged cache (adept_paged_attend).
//
// Tiles (head_dim 64 / 128): the (entry, query head) pairs that read one K/V head
// of one sequence are the columns of a matrix; a plan kernel cuts each sequence's
// columns into tiles of 128.  A workgroup takes one (tile, K/V head) and, where
// there are too few of those to fill the card, a part of the keys, which a second
// kernel joins.  Bound by the matrix cores and the waves' issue beside them together.
//
// Steps (head_dim 64 / 128, bf16, one entry per sequence): a workgroup takes a
// stretch of one entry's keys for one K/V head; a second kernel joins the
// stretches of an entry.  Bound by HBM.
//
// Walk (other widths): one wave per (entry, head) takes the keys one after
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
#include "paged_cut.h"

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
    const int s = c.slot(pages[t >> c.shift], t, true);
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
// on, G columns each): columns col .. col + cols - 1, cols <= TC_ (0: no tile).
struct Tile {
  int first, col, cols, seq;
};

// Segments: stretches of entries of one sequence.  Each pass takes 8 entries of
// every thread, all loads of the pass in flight together, and ranks the starts by
// wave ballots; then a scan over the segments' tile counts.  starts:
// [max_active + 1].  One workgroup, whose chain of loads is what it takes: 4 us for
// 500 entries, 14 for 16384.  (The entries' limits and the tiles' ends formed here
// too, to shorten the start of the tiles' workgroups: 8 and 29 us, and no more won.)
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(
    Entries e, int G, int max_tiles, int32_t* __restrict__ starts, Tile* __restrict__ tiles,
    int32_t* __restrict__ n_tiles) {
  constexpr int U = 8, W = kPlanThreads / 64;
  __shared__ int cnt[U * W], base_s, nt_s;
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
      const int k = k0 + u * kPlanThreads + tid;
      m[u] = __ballot(k < n && at[u] != before[u]);
      if (lane == 0) cnt[u * W + wave] = __popcll(m[u]);
    }
    __syncthreads();
    if (wave == 0) {               // exclusive ranks of the U * W counts
      constexpr int P = U * W / 64;
      int c4[P], sum = 0;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        c4[i] = sum;
        sum += cnt[P * lane + i];
      }
      int x = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
      }
      const int base = base_s + x - sum;
#pragma unroll
      for (int i = 0; i < P; ++i) cnt[P * lane + i] = base + c4[i];
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
  if (wave == 0) {                 // the segments' tiles, 64 segments at a time
    int acc = 0;
    for (int i0 = 0; i0 < ns; i0 += 64) {
      const int i = i0 + lane;
      const int first = i < ns ? starts[i] : 0, next = i < ns ? starts[i + 1] : 0;
      const int64_t cols = (int64_t)(next - first) * G;
      const int mine = (int)((cols + TC_ - 1) / TC_);
      const int seq = i < ns ? e.seq[e.rows[first]] : 0;
      // all first tiles, all second ones, ...: those of the same place in their
      // prompts next to each other
      for (int t = 0;; ++t) {
        const uint64_t more = __ballot(mine > t);
        if (more == 0) break;
        if ((more & (more - 1)) == 0) {      // one segment's rest: a lane a tile
          const int j = __ffsll((unsigned long long)more) - 1;
          const int f = __builtin_amdgcn_readlane(first, j), b = __builtin_amdgcn_readlane(seq, j);
          const int nj = __builtin_amdgcn_readlane(mine, j);
          const int64_t cj = (int64_t)(__builtin_amdgcn_readlane(next, j) - f) * G;
          for (int u = t + lane; u < nj; u += 64)
            tiles[acc + u - t] = Tile{f, u * TC_, (int)min((int64_t)TC_, cj - (int64_t)u * TC_), b};
          acc += nj - t;
          break;
        }
        if (mine > t)
          tiles[acc + __popcll(more & ((1ull << lane) - 1))] =
              Tile{first, t * TC_, (int)min((int64_t)TC_, cols - (int64_t)t * TC_), seq};
        acc += __popcll(more);
      }
    }
    if (lane == 0) {
      *n_tiles = acc;
      nt_s = acc;
    }
  }
  __syncthreads();
  const int nt = nt_s;
  for (int t = nt + tid; t < max_tiles; t += kPlanThreads) tiles[t] = Tile{0, 0, 0, 0};
}

// ---------------------------------------------------------------------------
// tiles
// ---------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
constexpr float kLazy = 8.0f;   // log2 headroom of the reference maximum
constexpr int KB = 64;          // keys of a block
constexpr int kTileThreads = 256;

// What takes the place of the K and V rows of keys that no column sees.
__device__ const uint4 kZeroRow[16] = {};

// max(a, b, c) without quieting the matrix products' results first (fmaxf
// would: one more instruction a value).  The compiler does not see that this
// reads a product's result and puts no wait for it: the first maximum over a
// product's result is taken by fmaxf, the others depend on it.
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
__device__ __forceinline__ float max_column(float m) {   // over lanes l, l^16, l^32, l^48
  const uint32_t u = __float_as_uint(m);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return max_halves(max3_raw(m, __uint_as_float(a[0]), __uint_as_float(a[1])));
}
__device__ __forceinline__ void store4(bf16* p, float a, float b, float c, float d) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}
__device__ __forceinline__ bool finite(float x) {
  return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u;
}

// Direct loads: 16 bytes of each lane to LDS, lane l's at dst + 16 l (dst: a uniform
// LDS address), from an address of each lane or from a uniform one and a byte
// offset of each lane.  Waited for by wait_loads(): the compiler, where it knows of
// such a load, puts a wait for all of them in front of every transposing LDS read.
// m0 is named as overwritten, so that nothing of the compiler's stays in it (it
// warns that a reserved register keeps no value across the block, as is meant).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds16(const char* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(dst)
               : "memory", "m0");
}
__device__ __forceinline__ void load_lds16(const char* base, uint32_t off, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off),
               "s"(base), "s"(dst)
               : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(
      __attribute__((address_space(3))) const char*)p);
}
// The lane number, in a way that keeps what is formed from it where it is used
// (not in registers across a loop that has none to spare).
__device__ __forceinline__ int lane_here() {
  int l = threadIdx.x & 63;
  asm volatile("" : "+v"(l));
  return l;
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Between a wave's LDS writes and its reads of what other lanes wrote (and the
// other way round): the hardware keeps a wave's LDS accesses in order, this keeps
// the compiler from changing it.  No instruction.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// (m, l, o) += the same of other keys; m in the exp2 domain.  Parts without keys
// have l = 0 and o = 0.
__device__ __forceinline__ void join(float& m, float& l, f32x4_t& o, float m2, float l2, f32x4_t o2) {
  const float mn = fmaxf(m, m2);
  const float a = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
  const float b = m2 == mn ? 1.0f : __builtin_amdgcn_exp2f(m2 - mn);
  m = mn;
  l = fmaf(b, l2, l * a);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = fmaf(b, o2[i], o[i] * a);
}

// Column j of a tile: its entry and query head.
__device__ __forceinline__ void column_of(const Tile& t, int j, int G, int hk, int* k, int* h) {
  const int c = t.col + j;
  *k = t.first + c / G;
  *h = hk * G + c % G;
}

// Work item of a workgroup, head by head: tile (-1: none), K/V head, part of the
// keys.  The hardware deals workgroups round-robin to the 8 XCDs: with 8 K/V heads or more each XCD takes a run of
// items, so that the tiles in flight on it share a few heads' K/V in its L2;
// with fewer heads the items are dealt as they come, which keeps the XCDs evenly
// loaded.
struct TileItem {
  int tile, head, part;
  bool whole;      // takes all of its tile's keys
};
__device__ __forceinline__ TileItem tile_item(int max_tiles, int heads, int parts, int nt) {
  const int total = max_tiles * heads * parts;
  int item = blockIdx.x;
  if (heads >= 8) {
    const int per = (total + 7) >> 3;
    item = (int)(blockIdx.x >> 3) < per ? (blockIdx.x & 7) * per + (blockIdx.x >> 3) : total;
  }
  // the last tiles first: of prompts, the longest
  TileItem t{max_tiles - 1 - item / parts % max_tiles, item / parts / max_tiles, item % parts,
             parts == 1};
  // a list whose sequences are scattered can hold more tiles than the host
  // counted on: then each workgroup takes several, with all of their keys
  if (nt > max_tiles) t.whole = true;
  if (item >= total || (t.whole && t.part > 0)) t.tile = -1;
  return t;
}
// The limits of the tile's columns: *n: keys that some column sees (0 .. *n - 1);
// returns column j's.  Every wave reads all columns' (two a lane).
__device__ __forceinline__ int tile_limits(const Entries& e, const PagedView& c, const Tile& tile,
                                           int G, int hk, int j, int* n) {
  static_assert(TC_ == 128, "two columns a lane");
  const int lane = threadIdx.x & 63;
  int row[2], lim[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int k, h;
    column_of(tile, min(lane + 64 * i, tile.cols - 1), G, hk, &k, &h);
    row[i] = e.rows[k];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int b;
    lim[i] = entry_limit(e, c, row[i], &b);     // columns past the last repeat it
  }
  int m = max(lim[0], lim[1]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, __shfl_xor(m, o, 64));
  *n = __builtin_amdgcn_readfirstlane(m);
  const int a = __shfl(lim[0], j & 63, 64), b = __shfl(lim[1], j & 63, 64);
  return j >= tile.cols ? 0 : j < 64 ? a : b;
}

// One workgroup per (tile, K/V head, part of the keys).  Wave w holds columns
// 32 w .. 32 w + 31.  Scores come transposed, S^T = K Q^T (32 keys x 32 columns,
// v_mfma_f32_32x32x16_bf16): lanes l and l + 32 hold one column's scores, the
// first the keys 8 i + 0 .. 3, the second 8 i + 4 .. 7, so a column's maximum
// takes one lane swap, and the weights already lie as the B operand of
// O^T += V^T P^T wants them, if V^T is read in the same order of keys.
//
// K and V come in blocks of 64 keys, bf16 in LDS.  A wave works on 32 keys at a
// time: the scores of the next 32 are formed beside the exponentials of these (a
// matrix instruction runs 32 cycles and takes 4 to issue), then these are
// multiplied into the output.  So K of block kb + 1 is needed before V of block kb
// is done with: two stages of K, three of V, one barrier a block, block kb + 2 on
// its way while block kb + 1 is computed.  Bound by neither unit alone: a 64-key block
// of a wave takes some 2400 cycles of its SIMD (counters: 500 tokens over 7900 in 8
// bits 2380, 8 prompts of 2048 in bf16 2500), 1024 of them matrix instructions.  A
// wave issues 2100 cycles a block itself (vector units 1200, the exponentials among
// them, LDS 220 .. 380, scalar 360 .. 520), which the other wave of the SIMD only partly
// overlaps: it waits for an issue slot 28 % of its time, for LDS, loads and the barrier
// about as long; and no wave is there for 8 .. 15 % of the time, before and behind the
// workgroups.  37 % of the matrix cores' cycles in all.  8 prompts of 2048 tokens, 32
// heads of 128: 365 us with the plan (0.75 PFLOP/s); 500 tokens over 7900 in 8 bits,
// 64/8 heads: 163 us with the join (0.82).  Waves of 64 columns, which read each
// fragment for two products but leave a SIMD one wave: 503 us for the 8 prompts.  The
// kernels for 128 dims spill 2 and 28 registers (8 bits), outside the loop over keys.
//
// A bf16 cache is copied to LDS by direct loads; an 8-bit one goes through
// registers, where its codes become bf16 with their scale in the conversion itself
// (exactly).  The slot of key t0 + lane is found by every wave from a page read a
// block earlier (read where it is needed its wait would be one for all loads on
// their way: 15 % more time when that was measured); its ballot is the mask of the
// keys that are there, and the others' rows are read from a row of zeros, so that
// they add nothing whatever the cache holds.
//
// Chunk c (16 bytes) of row r lies at c ^ fk(r) in K, c ^ fv(r) in V: the K
// reads (32 rows, two chunks) and the transposing V reads (4 rows, 4 chunks in
// each half) then fall on distinct banks.
template <int HD, bool FP8>
__global__ __launch_bounds__(kTileThreads, 2) void paged_tile_kernel(
    int H, float scale_log2, const bf16* __restrict__ q, Entries e, PagedView c,
    const Tile* __restrict__ tiles, const int32_t* __restrict__ n_tiles,
    int max_tiles, int parts, bf16* __restrict__ out,
    float* __restrict__ part) {
  constexpr int DS = HD / 16;               // 16-dim steps of S
  constexpr int DB = HD / 32;               // 32-dim blocks of O^T
  constexpr int ROWB = HD * 2;              // bytes of a row in LDS
  constexpr int NCH = ROWB / 16;            // its 16-byte chunks
  constexpr int RPI = 1024 / ROWB;          // rows of one direct load of a wave
  constexpr int DPW = KB / RPI / 4;         // direct loads of a wave and operand
  constexpr int BLK = KB * ROWB;
  constexpr int NCO = ROWB / 16;            // chunks of a row of the output
  // 8-bit cache: 16-byte pieces of a row, and how many of a block a thread takes
  constexpr int PCH = HD / 16, PPT = KB * PCH / kTileThreads;
  __shared__ __attribute__((aligned(1024))) char sK[2][BLK], sV[3][BLK];

  const int G = H / c.n_kv_heads;
  const int nt = *n_tiles;
  const TileItem it = tile_item(max_tiles, c.n_kv_heads, parts, nt);
  if (it.tile < 0) return;
  const int hk = it.head, p = it.part;
  const bool whole = it.whole;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, c32 = lane & 31;
  auto fk = [](int r) { return HD == 128 ? (r & 15) : ((r >> 1) & 7); };
  auto fv = [](int r) { return HD == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); };

  for (int ti = it.tile; ti < nt; ti += max_tiles) {
    const Tile tile = tiles[ti];
    if (tile.cols == 0) return;
    const int32_t* pages = c.table + (int64_t)tile.seq * c.max_pages;
    const int j = wave * 32 + c32;
    const bool valid = j < tile.cols;
    int tend;
    const int qlim = tile_limits(e, c, tile, G, hk, j, &tend);
    const KeyRange range = part_of_keys(tend, whole ? 1 : parts, p, KB);
    const int tb = range.begin, te = range.end;
    const int nkb = (te - tb + KB - 1) / KB;
    auto key_of = [&](int kb) { return tb + kb * KB + lane; };
    auto page_of = [&](int kb) { return pages[min(key_of(kb), te - 1) >> c.shift]; };
    int page = nkb > 0 ? page_of(0) : 0;
    int qk, qh;
    column_of(tile, valid ? j : 0, G, hk, &qk, &qh);
    const int64_t qat = ((int64_t)qk * H + qh) * HD;

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

    // slots of a block's keys, one per lane; block kb + 1's pages are read during block kb - 1
    auto slots_of = [&](int kb, int page) { return c.slot(page, key_of(kb), key_of(kb) < te); };
    const int64_t rowc = (int64_t)c.n_kv_heads * HD;    // elements of a slot
    // Where a load's rows lie in one page and are all there, its address is a
    // uniform base and fixed offsets of the lanes (else some 100 instructions a
    // block, as many as the softmax takes).
    constexpr int RUN = 64 / (FP8 ? PCH : NCH);         // rows of a wave's load
    const bool runs = (1 << c.shift) >= RUN;
    const uint32_t rowb = (uint32_t)(rowc * (FP8 ? 1 : 2));
    auto base_of = [&](int op, int s) {
      return (const char*)(op ? c.v : c.k) + s * (int64_t)rowb + hk * HD * (FP8 ? 1 : 2);
    };
    // bf16: direct loads
    // (lane offsets: load jj's K rows lie 4 jj chunks further in fk, fv repeats
    // every RPI rows)
    const uint32_t koff = (lane / NCH) * rowb + ((lane % NCH) ^ fk(lane / NCH)) * 16;
    const uint32_t voff = (lane / NCH) * rowb + ((lane % NCH) ^ fv(lane / NCH)) * 16;
    const uint32_t ldsK = lds_address(sK), ldsV = lds_address(sV);
    auto issue_run = [&](int jj, uint32_t ko, uint32_t vo, int sl) {
      const int qd = wave * DPW + jj, s = __builtin_amdgcn_readlane(sl, qd * RPI);
      load_lds16(base_of(0, s), koff ^ (64 * jj), ldsK + ko + qd * 1024);
      load_lds16(base_of(1, s), voff, ldsV + vo + qd * 1024);
    };
    auto issue = [&](uint32_t ko, uint32_t vo, int sl) {
#pragma unroll
      for (int jj = 0; jj < DPW; ++jj) {
        const int qd = wave * DPW + jj;
        const uint32_t dst[2] = {ldsK + ko + qd * 1024, ldsV + vo + qd * 1024};
        const int l = lane_here(), r = qd * RPI + l / NCH;
        const int s = __shfl(sl, r, 64);
#pragma unroll
        for (int op = 0; op < 2; ++op)
          load_lds16((s < 0 ? (const char*)kZeroRow : base_of(op, s)) +
                         ((l % NCH) ^ (op ? fv(r) : fk(r))) * 16,
                     dst[op]);
      }
    };
    // 8-bit: codes and scales to registers, then as bf16 to LDS
    u32x4_t code[2][PPT];
    uint8_t csc[2][PPT];
    auto fetch = [&](int sl, bool all) {
#pragma unroll
      for (int i = 0; i < PPT; ++i) {
        const int l = lane_here(), r = i * (kTileThreads / PCH) + wave * RUN + l / PCH;
        const int s = all ? __builtin_amdgcn_readlane(sl, i * (kTileThreads / PCH) + wave * RUN)
                          : max(__shfl(sl, r, 64), 0);
#pragma unroll
        for (int op = 0; op < 2; ++op) {
          const uint8_t* sc = op ? c.v_scale : c.k_scale;
          if (all) {
            code[op][i] = *reinterpret_cast<const u32x4_t*>(
                base_of(op, s) + ((l / PCH) * rowb + l % PCH * 16));
            csc[op][i] = (sc + (int64_t)s * c.n_kv_heads + hk)[(l / PCH) * (uint32_t)c.n_kv_heads];
          } else {
            code[op][i] = *reinterpret_cast<const u32x4_t*>(base_of(op, s) + l % PCH * 16);
            csc[op][i] = sc[(int64_t)s * c.n_kv_heads + hk];
            // not there: zeros, with a scale of their own (0 times slot 0's may be NaN)
            if (__shfl(sl, r, 64) < 0) {
              code[op][i] = u32x4_t{0, 0, 0, 0};
              csc[op][i] = kScaleOne;
            }
          }
        }
      }
    };
    auto put = [&](uint32_t ko, uint32_t vo) {
#pragma unroll
      for (int i = 0; i < PPT; ++i) {
        const int pc = i * kTileThreads + tid, r = pc / PCH;
#pragma unroll
        for (int op = 0; op < 2; ++op) {
          char* row = (op ? &sV[0][0] + vo : &sK[0][0] + ko) + r * ROWB;
          const float sc = scale_of(csc[op][i]);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t a = code[op][i][2 * half], b = code[op][i][2 * half + 1];
            const int ch = (pc % PCH * 2 + half) ^ (op ? fv(r) : fk(r));
            *reinterpret_cast<u32x4_t*>(row + ch * 16) =
                u32x4_t{fp8x2_to_bf16x2<false>(a, sc), fp8x2_to_bf16x2<true>(a, sc),
                        fp8x2_to_bf16x2<false>(b, sc), fp8x2_to_bf16x2<true>(b, sc)};
          }
        }
      }
    };

    // block kb: its loads, from the slots of its keys; `there` is their mask.  Those
    // of a bf16 block whose loads are runs are left to the step (returns true): eight
    // in a row would hold the wave for some 800 cycles.
    uint64_t there = 0;
    int sl = -1;
    auto load = [&](int kb, uint32_t ko, uint32_t vo) {
      sl = slots_of(kb, page);
      there = __ballot(sl >= 0);
      page = page_of(kb + 1);
      const bool run = runs && there == ~0ull;
      if constexpr (FP8) {
        if (run) fetch(sl, true); else fetch(sl, false);
        return false;
      } else {
        if (!run) issue(ko, vo, sl);
        return run;
      }
    };
    auto landed = [&](uint32_t ko, uint32_t vo) {
      if constexpr (FP8) put(ko, vo); else wait_loads();
    };
    // LDS addresses of this lane's fragments: K step ds at ka ^ 32 ds (fk only
    // touches the chunk bits), V^T block db at va ^ 64 db
    typedef __attribute__((address_space(3))) const bf16x8_t lds_bf16x8;
    const int r0 = 4 * hh + ((lane & 15) >> 2);
    const uint32_t ka0 = ldsK + c32 * ROWB + ((hh ^ fk(c32)) * 16);
    const uint32_t va0 = ldsV + r0 * ROWB +
                         (fv(r0) + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 + 8 * (lane & 1);
    auto read_k = [&](uint32_t ka, int ds) { return *(lds_bf16x8*)(uintptr_t)(ka ^ (32 * ds)); };
    // scores of 32 keys
    auto scores = [&](uint32_t ka, f32x16_t& s) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = 0.0f;
#pragma unroll
      for (int ds = 0; ds < DS; ++ds)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_k(ka, ds), qf[ds], s, 0, 0, 0);
    };
    auto column_max = [&](const f32x16_t& s) {
      float m = fmaxf(s[0], s[1]);
#pragma unroll
      for (int v = 2; v < 16; v += 2) m = max3_raw(m, s[v], s[v + 1]);
      return m;
    };
    // the reference maximum moves (and o is rescaled) only where new scores
    // exceed it by more than 2^kLazy
    auto raise = [&](float m) {
      if (!__any(m * scale_log2 > m_ref + kLazy)) return;
      const float mb = max_halves(m) * scale_log2;
      const float mn = fmaxf(m_ref, mb);
      const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_ref - mn);
      m_ref = mn;
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[i][v] *= alpha;
    };
    // V^T fragments of dim block db and 32 keys: in each 16-lane group source lane
    // L reads 4 dims of key k0 + L/4 and lane i receives dim n0 + i of keys k0 ..
    // k0 + 3
    auto read_v = [&](uint32_t va, int db, bf16x8_t (&a)[2]) {
      const uint32_t at = va ^ (64 * db);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s16x4 half[2];
#pragma unroll
        for (int x = 0; x < 2; ++x)     // fv repeats every 4 rows
          half[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_s16x4*)(uintptr_t)(at + (16 * i + 8 * x) * ROWB));
        a[i] = __builtin_bit_cast(bf16x8_t,
                                  __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
      }
    };
    // One step of the pipeline: the scores `sn` of the next 32 keys (K at ka) beside
    // the weights of these 32 (scores sc), two exponentials to a product; then these
    // into the output (V at va) beside the maximum of sn, which is returned.  The
    // weights are rounded to bf16 for the product, as adept_attend's are (the sum takes
    // the rounded ones, so that they still add up to one): at most 2^-8 of a weight,
    // 0.0019 of the result against 64 bits where its own rounding alone makes 0.0016.
    // Weights of 16 bits, by a second product for what the first leaves, were measured:
    // 0.0016, for 495 us instead of 364 (8 x 2048), 212 instead of 163 (1 x 500).
    // run: loads on the way, one pair to a product.  Of the two waves of a SIMD the
    // one in a step goes first where the other one converts codes or sets out (1 x
    // 500 over 8 bits 161 us, 167 without; 5 x 250 heads of 64 22.8, 23.6; bf16 of
    // 128, whose waves do little else, 370 either way).
    auto step = [&](bool run, uint32_t ka, f32x16_t& sn, uint32_t va, const f32x16_t& sc,
                    uint32_t ko, uint32_t vo) {
      constexpr int AHEAD = 3, EPS = 16 / DS;    // fragments read ahead, weights of a product
      constexpr bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};
      const float msub = m_ref == -INFINITY ? 0.0f : m_ref;
      bf16x8_t a[DS], v[2][2];
#pragma unroll
      for (int ds = 0; ds < AHEAD; ++ds) a[ds] = read_k(ka, ds);
      if constexpr (FP8 || HD == 64) __builtin_amdgcn_s_setprio(1);
      uint32_t w[8];
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) {
        if (ds == 0)
#pragma unroll
          for (int x = 0; x < 16; ++x) sn[x] = 0.0f;
        sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[ds], qf[ds], sn, 0, 0, 0);
        if (ds + AHEAD < DS) a[ds + AHEAD] = read_k(ka, ds + AHEAD);
        if (ds == DS - 2) read_v(va, 0, v[0]);
#pragma unroll
        for (int x = ds * EPS; x < (ds + 1) * EPS; x += 2) {
          w[x / 2] = pack_bf16x2(__builtin_amdgcn_exp2f(fmaf(sc[x], scale_log2, -msub)),
                                 __builtin_amdgcn_exp2f(fmaf(sc[x + 1], scale_log2, -msub)));
          l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[x / 2]), ones,
                                                  l_run, false);
        }
        if constexpr (!FP8)
          if (run && ds % (DS / DPW) == DS / DPW - 1) issue_run(ds / (DS / DPW), ko, vo, sl);
        __builtin_amdgcn_sched_barrier(0);
      }
      bf16x8_t pb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        pb[i] = __builtin_bit_cast(
            bf16x8_t, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
      float m = 0.0f;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        if (db + 1 < DB) read_v(va, db + 1, v[(db + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[db & 1][i], pb[i], o[db], 0, 0, 0);
#pragma unroll
        for (int x = db * (16 / DB); x < (db + 1) * (16 / DB); x += 2)
          m = x == 0 ? fmaxf(sn[0], sn[1]) : max3_raw(m, sn[x], sn[x + 1]);
      }
      if constexpr (FP8 || HD == 64) __builtin_amdgcn_s_setprio(0);
      return m;
    };

    uint64_t mask = 0, mask1 = 0;      // of blocks kb and kb + 1
    f32x16_t s[2];
    if (nkb > 0) {
      if (load(0, 0, 0))
#pragma unroll
        for (int jj = 0; jj < DPW; ++jj) issue_run(jj, 0, 0, sl);
      mask = there;
    }
    int wend = qlim, wfull = valid ? qlim : INT_MAX;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      wend = max(wend, __shfl_xor(wend, o, 64));
      wfull = min(wfull, __shfl_xor(wfull, o, 64));
    }
    wend = __builtin_amdgcn_readfirstlane(wend);     // the wave's columns see keys below it,
    wfull = __builtin_amdgcn_readfirstlane(wfull);   // and all of them the ones below this
    // waited for here: a wait inside the loop would be one for the loads on their way
#pragma unroll
    for (int s = 0; s < DS; ++s) asm volatile("" : "+v"(qf[s]));
    // keys past a column's end, or that are not there; m: the maximum, then formed again
    auto hide = [&](int t0, uint64_t mask, int kt, f32x16_t& s, float& m) {
      if (t0 + KB <= wfull && mask == ~0ull) return;
      const int h4 = 4 * (lane_here() >> 5);
      const int lim = qlim - t0 - kt * 32 - h4;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = 8 * (v >> 2) + (v & 3) < lim ? s[v] : -INFINITY;
      if (mask != ~0ull) {
        const uint32_t mk = (uint32_t)(mask >> (kt * 32)) >> h4;
#pragma unroll
        for (int v = 0; v < 16; ++v)
          s[v] = mk & (1u << (8 * (v >> 2) + (v & 3))) ? s[v] : -INFINITY;
      }
      m = column_max(s);
    };
    constexpr uint32_t HALF = 32 * ROWB;
    if (nkb > 0) {
      landed(0, 0);
      __syncthreads();
      if (nkb > 1 && load(1, BLK, BLK))
#pragma unroll
        for (int jj = 0; jj < DPW; ++jj) issue_run(jj, BLK, BLK, sl);
      mask1 = there;
      if (tb < wend) {
        scores(ka0, s[0]);
        float m = column_max(s[0]);
        hide(tb, mask, 0, s[0], m);
        raise(m);
      }
    }
    uint32_t vo = 0, von = BLK;        // of block kb's V and of block kb + 1's
    for (int kb = 0; kb < nkb; ++kb) {
      const int t0 = tb + kb * KB;
      const uint32_t ko = (kb & 1) * BLK, von2 = von == 2 * BLK ? 0 : von + BLK;
      if (t0 < wend) {     // a wave whose columns have seen their keys only loads
        float m = step(false, ka0 + ko + HALF, s[1], va0 + vo, s[0], 0, 0);
        hide(t0, mask, 1, s[1], m);
        raise(m);
      }
      if (kb + 1 < nkb) landed(ko ^ BLK, von);
      __syncthreads();     // block kb + 1 is in LDS; K of kb and V of kb - 1 are free
      const bool run = kb + 2 < nkb && load(kb + 2, ko, von2);
      if (t0 + 32 < wend) {
        // (behind the last block: scores that are not used)
        const uint32_t ka = ka0 + (ko ^ BLK), va = va0 + vo + HALF;
        float m = step(run, ka, s[0], va, s[1], ko, von2);
        hide(t0 + KB, mask1, 0, s[0], m);
        if (kb + 1 < nkb) raise(m);
      } else if (run) {
#pragma unroll
        for (int jj = 0; jj < DPW; ++jj) issue_run(jj, ko, von2, sl);
      }
      mask = mask1;
      mask1 = there;
      vo = von;
      von = von2;
    }

    const float l = l_run + __shfl_xor(l_run, 32, 64);
    float zero = l * 0.0f;             // NaN where l or an o is not finite
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) zero = fmaf(o[i][v], 0.0f, zero);
    const uint64_t bad = __ballot(valid && zero != 0.0f);
    const uint32_t redo = (uint32_t)bad | (uint32_t)(bad >> 32);   // by column
    float* pp = nullptr;     // this column's partial result: m, l, then the dims
    if (!whole) pp = part + (((int64_t)ti * c.n_kv_heads + hk) * parts + p) * TC_ * (HD + 2);
    if (whole) {
      // turned round in LDS (the wave's own 32 rows, chunk c of row r at c ^ f(r)),
      // so that whole rows are written
      __syncthreads();                 // V is read
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      char* row = &sV[0][0] + (wave * 32 + c32) * ROWB;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *reinterpret_cast<uint2*>(row + ((db * 4 + v / 4) ^ (c32 & (NCO - 1))) * 16 + 8 * hh) =
              make_uint2(pack_bf16x2(o[db][v] * inv, o[db][v + 1] * inv),
                         pack_bf16x2(o[db][v + 2] * inv, o[db][v + 3] * inv));
      wave_lds_order();
#pragma unroll
      for (int i = 0; i < 32 * NCO / 64; ++i) {
        const int r = i * (64 / NCO) + lane / NCO, ch = lane % NCO;
        const int64_t at = __shfl((long long)qat, r, 64);
        const uint4 y = *reinterpret_cast<const uint4*>(
            &sV[0][0] + (wave * 32 + r) * ROWB + (ch ^ (r & (NCO - 1))) * 16);
        if (wave * 32 + r < tile.cols && !((redo >> r) & 1))
          *reinterpret_cast<uint4*>(out + at + ch * 8) = y;
      }
    } else if (valid && !((redo >> c32) & 1)) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *reinterpret_cast<float4*>(pp + TC_ * 2 + j * HD + db * 32 + 2 * v + 4 * hh) =
              make_float4(o[db][v], o[db][v + 1], o[db][v + 2], o[db][v + 3]);
      if (hh == 0) *reinterpret_cast<float2*>(pp + 2 * j) = make_float2(m_ref, l);
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
template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_tile_join_kernel(
    int H, int n_kv_heads, const Tile* __restrict__ tiles,
    const int32_t* __restrict__ n_tiles, int max_tiles, int parts, const float* __restrict__ part,
    T* __restrict__ out) {
  constexpr int CPB = 256 / (HD / 4);      // columns of a workgroup
  const int ti = blockIdx.x, hk = blockIdx.y, nt = *n_tiles;
  if (ti >= nt || nt > max_tiles) return;      // (more: nothing was cut)
  const Tile tile = tiles[ti];
  const int G = H / n_kv_heads;
  const int j = blockIdx.z * CPB + threadIdx.x / (HD / 4), d = threadIdx.x % (HD / 4) * 4;
  if (j >= tile.cols) return;
  const float* pp = part + ((int64_t)ti * n_kv_heads + hk) * parts * TC_ * (HD + 2);
  float m = -INFINITY, l = 0.0f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const float* x = pp + (int64_t)p * TC_ * (HD + 2);
    const float2 ml = *reinterpret_cast<const float2*>(x + 2 * j);
    join(m, l, o, ml.x, ml.y, *reinterpret_cast<const f32x4_t*>(x + TC_ * 2 + j * HD + d));
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  int k, h;
  column_of(tile, j, G, hk, &k, &h);
  store4(out + ((int64_t)k * H + h) * HD + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
}

// ---------------------------------------------------------------------------
// tiles of f32 queries
// ---------------------------------------------------------------------------
constexpr int kTile32Threads = 512;
constexpr int KB32 = 32;

// As paged_tile_kernel, in f32 throughout (v_mfma_f32_16x16x4_f32): eight waves of
// 16 columns, blocks of 32 keys in one stage of LDS, the next block's rows in
// registers while a block is computed.  A score tile is 16 keys x 16 columns;
// lane (g, c) holds the keys 4 g + 0 .. 3 of column c, so product v of
// O^T += V^T P^T takes the keys 4 g + v from its register v as they are.  Bound by
// the f32 matrix rate (1/16 of bf16's), small calls by their launches.
template <int HD, bool FP8>
__global__ __launch_bounds__(kTile32Threads) void paged_tile_f32_kernel(
    int H, float scale_log2, const float* __restrict__ q, Entries e, PagedView c,
    const Tile* __restrict__ tiles, const int32_t* __restrict__ n_tiles,
    int max_tiles, int parts, float* __restrict__ out,
    float* __restrict__ part) {
  constexpr int DB = HD / 16;
  constexpr int ROW = HD;                            // floats of a row in LDS
  constexpr int NCH = HD * (FP8 ? 1 : 4) / 16;       // 16-byte pieces of a cache row
  constexpr int PPT = (KB32 * NCH + kTile32Threads - 1) / kTile32Threads;   // of a thread
  __shared__ __attribute__((aligned(16))) float sKV[2][KB32 * ROW];
  const int G = H / c.n_kv_heads;
  const int nt = *n_tiles;
  const TileItem it = tile_item(max_tiles, c.n_kv_heads, parts, nt);
  if (it.tile < 0) return;
  const int hk = it.head, p = it.part;
  const bool whole = it.whole;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  // 16-byte chunk ch of row r lies at ch ^ f(r): the reads of K (16 rows, a
  // chunk) and of V (4 rows four apart, 64 bytes) fall on distinct banks
  auto fk = [](int r) { return r & 15; };
  auto fv = [](int r) { return 4 * ((r >> 2) & 3); };

  for (int ti = it.tile; ti < nt; ti += max_tiles) {
    const Tile tile = tiles[ti];
    if (tile.cols == 0) return;
    const int32_t* pages = c.table + (int64_t)tile.seq * c.max_pages;
    const int j = wave * 16 + c16;
    const bool valid = j < tile.cols;
    int qk, qh;
    column_of(tile, valid ? j : 0, G, hk, &qk, &qh);
    const int64_t qat = ((int64_t)qk * H + qh) * HD;
    int tend;
    const int qlim = tile_limits(e, c, tile, G, hk, j, &tend);
    int wend = qlim;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) wend = max(wend, __shfl_xor(wend, o, 64));
    wend = __builtin_amdgcn_readfirstlane(wend);
    const KeyRange range = part_of_keys(tend, whole ? 1 : parts, p, KB);
    const int tb = range.begin, te = range.end;
    const int nkb = (te - tb + KB32 - 1) / KB32;

    f32x4_t qf[HD / 16];      // dims 16 i + 4 g + 0 .. 3
#pragma unroll
    for (int i = 0; i < HD / 16; ++i)
      qf[i] = *reinterpret_cast<const f32x4_t*>(q + qat + i * 16 + g * 4);
    f32x4_t o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_ref = -INFINITY, l_run = 0.0f;

    auto key_of = [&](int kb) { return tb + kb * KB32 + (lane & 31); };
    auto page_of = [&](int kb) { return pages[min(key_of(kb), te - 1) >> c.shift]; };
    const int64_t rowc = (int64_t)c.n_kv_heads * HD;
    u32x4_t x[2][PPT];
    uint8_t xs[2][PPT];
    uint32_t there = 0;
    // rows of keys that are not there: slot 0's, cleared on their way to LDS
    auto fetch = [&](int kb, int page) {
      const int sl = c.slot(page, key_of(kb), key_of(kb) < te);
      there = (uint32_t)__ballot(sl >= 0);
#pragma unroll
      for (int i = 0; i < PPT; ++i) {
        const int pc = i * kTile32Threads + tid, r = pc / NCH % KB32;
        const int s = max(__shfl(sl, r, 64), 0);
#pragma unroll
        for (int op = 0; op < 2; ++op) {
          const char* src = (const char*)(op ? c.v : c.k) + (s * rowc + hk * HD) * (FP8 ? 1 : 4);
          x[op][i] = *reinterpret_cast<const u32x4_t*>(src + pc % NCH * 16);
          if constexpr (FP8)
            xs[op][i] = (op ? c.v_scale : c.k_scale)[(int64_t)s * c.n_kv_heads + hk];
        }
      }
    };
    auto put = [&]() {
#pragma unroll
      for (int i = 0; i < PPT; ++i) {
        const int pc = i * kTile32Threads + tid, r = pc / NCH, ch = pc % NCH;
        if (r >= KB32) continue;
        const bool in = (there >> r) & 1;
#pragma unroll
        for (int op = 0; op < 2; ++op) {
          float* row = sKV[op] + r * ROW;
          const int f = op ? fv(r) : fk(r);
          if constexpr (FP8) {
            const float sc = scale_of(xs[op][i]);
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const float2 a = fp8x2_to_f32x2<false>(x[op][i][z], sc);
              const float2 b = fp8x2_to_f32x2<true>(x[op][i][z], sc);
              const f32x4_t y = in ? f32x4_t{a.x, a.y, b.x, b.y} : f32x4_t{0.f, 0.f, 0.f, 0.f};
              *reinterpret_cast<f32x4_t*>(row + ((4 * ch + z) ^ f) * 4) = y;
            }
          } else {
            *reinterpret_cast<u32x4_t*>(row + (ch ^ f) * 4) = in ? x[op][i] : u32x4_t{0, 0, 0, 0};
          }
        }
      }
    };
    int page = 0;
    if (nkb > 0) {
      page = page_of(0);
      fetch(0, page);
      page = page_of(1);
    }
    for (int kb = 0; kb < nkb; ++kb) {
      const int t0 = tb + kb * KB32;
      const uint32_t mask = there;
      put();
      __syncthreads();
      if (kb + 1 < nkb) {
        const int next = page;
        page = page_of(kb + 2);
        fetch(kb + 1, next);
      }
      if (t0 < wend) {
        f32x4_t s[2];
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
          s[sb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          const int r = sb * 16 + c16;
#pragma unroll
          for (int i = 0; i < HD / 16; ++i) {
            const f32x4_t a =
                *reinterpret_cast<const f32x4_t*>(sKV[0] + r * ROW + ((4 * i + g) ^ fk(r)) * 4);
#pragma unroll
            for (int z = 0; z < 4; ++z)
              s[sb] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[z], qf[i][z], s[sb], 0, 0, 0);
          }
        }
        float mb = -INFINITY;
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int kl = sb * 16 + 4 * g + v;
            s[sb][v] = t0 + kl < qlim && ((mask >> kl) & 1) ? s[sb][v] * scale_log2 : -INFINITY;
            mb = max3_raw(mb, s[sb][v], s[sb][v]);
          }
        mb = max_column(mb);
        const float mn = fmaxf(m_ref, mb);
        const float alpha = mn == m_ref ? 1.0f : __builtin_amdgcn_exp2f(m_ref - mn);
        const float msub = mn == -INFINITY ? 0.0f : mn;
        m_ref = mn;
        l_run *= alpha;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
          for (int v = 0; v < 4; ++v) o[i][v] *= alpha;
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            s[sb][v] = __builtin_amdgcn_exp2f(s[sb][v] - msub);
            l_run += s[sb][v];
          }
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int r = sb * 16 + 4 * g + v;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              const float a = sKV[1][r * ROW + (((4 * db + (c16 >> 2)) ^ fv(r)) * 4) + (c16 & 3)];
              o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, s[sb][v], o[db], 0, 0, 0);
            }
          }
      }
      __syncthreads();
    }
    float l = l_run;
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    bool ok = finite(l);
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) ok &= finite(o[i][v]);
    uint64_t bad = __ballot(valid && !ok);
    bad |= bad >> 32;
    const uint32_t redo = (uint32_t)(bad | (bad >> 16)) & 0xffffu;
    float* pp = nullptr;
    if (!whole) pp = part + (((int64_t)ti * c.n_kv_heads + hk) * parts + p) * TC_ * (HD + 2);
    if (valid && !((redo >> c16) & 1)) {
      const float f = whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
      float* dst = whole ? out + qat : pp + TC_ * 2 + j * HD;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        f32x4_t y = o[db];
#pragma unroll
        for (int v = 0; v < 4; ++v) y[v] *= f;
        *reinterpret_cast<f32x4_t*>(dst + db * 16 + g * 4) = y;
      }
      if (!whole && g == 0) *reinterpret_cast<float2*>(pp + 2 * j) = make_float2(m_ref, l);
    }
    for (uint32_t left = redo; left; left &= left - 1) {
      const int y = __ffs(left) - 1, jj = wave * 16 + y;
      int k, h;
      column_of(tile, jj, G, hk, &k, &h);
      const int lim = min(__shfl(qlim, y, 64), te);
      const int64_t at = ((int64_t)k * H + h) * HD;
      const auto w = walk_keys<float, typename std::conditional<FP8, uint8_t, float>::type, HD / 64>(
          q + at, HD, scale_log2, c, pages, hk, tb, lim);
      if (whole) {
        walk_store(w, HD, out + at);
      } else {
        for (int i = 0; i < HD / 64; ++i) pp[TC_ * 2 + jj * HD + lane + 64 * i] = w.o[i];
        if (lane == 0) *reinterpret_cast<float2*>(pp + 2 * jj) = make_float2(w.m, w.l);
      }
    }
  }
}

// Tiles that the host counts on, and the parts of the keys with which they make
// up to kParts workgroups, two a CU; a part keeps kPartKeys of the keys there may
// be (1 x 64 tokens over 700, 32/8 heads: 24 us, 29 with 64).  f32 tiles take
// longer, 2 us for 32 keys, and gain from shorter parts: 2 x 100 tokens over 300
// 21 us with parts of 64 keys, 35 with 256; one workgroup a CU.
constexpr int kParts = 512, kPartKeys = 256, kParts32 = 256, kPartKeys32 = 64;
struct TileShape {
  int max_tiles, cap_tiles, parts;
  size_t off_tiles, off_starts, off_part, bytes;
};
TileShape tile_shape(adept_dtype dt, const adept_paged_kv& kv, int n_heads, int max_active,
                     int n_seq, int max_pages) {
  const int64_t G = n_heads / kv.n_kv_heads, keys = (int64_t)max_pages * kv.page_size;
  TileShape t{};
  const int64_t full = max_active * G / TC_;
  t.max_tiles = (int)(full + std::min(n_seq, max_active));
  t.cap_tiles = (int)(full + max_active);
  const int64_t base = (int64_t)t.max_tiles * kv.n_kv_heads;
  const bool f32 = dt == ADEPT_F32;
  const int64_t slots = f32 ? kParts32 : kParts;      // workgroups that parts make up to
  const int64_t most = std::min<int64_t>(ceil_div(keys, f32 ? kPartKeys32 : kPartKeys), 32);
  t.parts = (int)std::max<int64_t>(1, std::min(slots / std::max<int64_t>(base, 1), most));
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  t.off_tiles = 256;
  t.off_starts = t.off_tiles + up((size_t)t.cap_tiles * sizeof(Tile));
  t.off_part = t.off_starts + up(((size_t)max_active + 1) * sizeof(int32_t));
  t.bytes = t.off_part;
  // Fewer tiles are cut into more parts: space for what any smaller call cuts, so
  // that a workspace serves every bound of the entries up to the one it was made for.
  if (most > 1)
    t.bytes += (size_t)std::min(slots, base * most) * TC_ * (kv.head_dim + 2) * sizeof(float);
  return t;
}

bool tiles_fit(const adept_paged_kv& kv) { return kv.head_dim == 64 || kv.head_dim == 128; }

// ---------------------------------------------------------------------------
// steps: one entry per sequence
// ---------------------------------------------------------------------------
constexpr int SK = 32;             // keys of a wave's block
constexpr int kStepUnit = 4 * SK;  // keys of a workgroup's block: the unit of the cut
constexpr int kStepEntries = 1024; // entries up to which long ones are cut
constexpr int SC = 16;             // columns
// Workgroups that a call is cut into, about: 40 uneven sequences (8 K/V heads)
// 119 us with 2048, 131 with 4096, 153 with 8192 (a workgroup starts with some
// five dependent loads); 64 sequences of 4096 keys, 32 heads, 653, 641 and 663 us.
constexpr int kStepItems = 2048;

// Item x of the call: a stretch of one entry's keys.  Every workgroup finds its
// own: entries of all workgroups' keys together, cut into about `want` stretches
// of equal length (whole units; an entry without keys is one), so that a batch of
// uneven lengths keeps the card evenly loaded.  All threads return the same.
struct Stretch {
  int k, part, parts, seq, t0, t1;
};
__device__ __forceinline__ Stretch step_stretch(const Entries& e, const PagedView& c, int n, int x,
                                                int want, int least) {
  constexpr int P = kStepEntries / 256;
  __shared__ long long s_sum[4];
  __shared__ int s_cnt[4], s_out[6];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (n > kStepEntries) {
    Stretch r{x, 0, 1, 0, 0, 0};
    if (x >= n) r.parts = 0;
    else r.t1 = entry_limit(e, c, e.rows[x], &r.seq);
    return r;
  }
  int lim[P], seq[P], units[P];
  long long sum = 0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int k = tid * P + i;
    lim[i] = k < n ? entry_limit(e, c, e.rows[k], &seq[i]) : 0;
    units[i] = (int)(((long long)lim[i] + kStepUnit - 1) / kStepUnit);
    sum += units[i];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (lane == 0) s_sum[wave] = sum;
  if (tid < 6) s_out[tid] = 0;
  __syncthreads();
  sum = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
  const int cut = stretch_units(sum, want, least);
  int cnt = 0;
#pragma unroll
  for (int i = 0; i < P; ++i)
    cnt += tid * P + i < n ? stretches(units[i], cut) : 0;
  int scan = cnt;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(scan, o, 64);
    if (lane >= o) scan += y;
  }
  if (lane == 63) s_cnt[wave] = scan;
  __syncthreads();
  int at = scan - cnt;
  for (int w = 0; w < wave; ++w) at += s_cnt[w];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int parts = tid * P + i < n ? stretches(units[i], cut) : 0;
    if (x >= at && x < at + parts) {
      s_out[0] = tid * P + i;
      s_out[1] = x - at;
      s_out[2] = parts;
      s_out[3] = seq[i];
      const long long t0 = (long long)(x - at) * cut * kStepUnit;
      s_out[4] = (int)t0;
      s_out[5] = (int)min((long long)lim[i], t0 + (long long)cut * kStepUnit);
    }
    at += parts;
  }
  __syncthreads();
  return Stretch{s_out[0], s_out[1], s_out[2], s_out[3], s_out[4], s_out[5]};
}

// One workgroup per (stretch of an entry's keys, K/V head, 16 of its query
// heads).  The query heads are the columns of 16x16x32 products (one of 16 where
// heads are not shared: the products cost a small part of the time that the
// keys take to arrive).  Wave w takes every fourth block of 32 keys from block w
// on, whole rows at a time (16 bytes a lane), through registers into the wave's own
// 32 rows of LDS: K, read back as the A operand of S^T = K Q^T, then V over it,
// read transposed as the A operand of O^T += V^T P^T; no barrier in the loop.
// The loads of the next block go out as soon as LDS has taken this one's, so a
// wave has a block in flight (16 KB, 8 KB in 8 bits) while it computes.  (K
// loaded as operands, 64 bytes of 16 rows at a
// time, halves of lines: 64 sequences of 4096 keys 770 us, 653 so.)
// The pages of the block after that are read then too, a whole block before their
// slots are needed (formed at once, which waits for every load before, 64 sequences
// of 4096 keys in 8 bits took half as long again; 355 us now, 6 TB/s).
// The four waves' results are joined in LDS; a stretch that is not all of its
// entry's keys leaves (m, l, o) for paged_step_join_kernel.
template <int HD, bool FP8>
__global__ __launch_bounds__(256, FP8 || HD == 64 ? 3 : 2) void paged_step_kernel(
    int H, int col_groups, int want, int least, float scale_log2, const bf16* __restrict__ q,
    Entries e, PagedView c, bf16* __restrict__ out, int2* __restrict__ spans,
    float* __restrict__ part) {
  constexpr int DS = HD / 32;                      // 32-dim steps of S
  constexpr int DB = HD / 16;                      // 16-dim blocks of O^T
  constexpr int ROWB = HD * 2;                     // bytes of a V row in LDS
  constexpr int ESZ = FP8 ? 1 : 2;
  constexpr int NCH = HD * ESZ / 16;               // 16-byte pieces of a cache row
  constexpr int RPI = 64 / NCH;                    // rows of one load of a wave
  constexpr int RI = SK / RPI;                     // loads of K, and of V
  __shared__ __attribute__((aligned(16))) char s_rows[4][SK * ROWB];
  __shared__ float s_m[4][SC], s_l[4][SC];
  const int items = gridDim.x / (c.n_kv_heads * col_groups);   // stretches side by side
  const int x = blockIdx.x % items, hk = blockIdx.x / items % c.n_kv_heads,
            cg = blockIdx.x / items / c.n_kv_heads;
  const int n = min(*e.n_active, e.max_active);
  const Stretch st = step_stretch(e, c, n, x, want, least);
  if (st.parts == 0) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  const int G = H / c.n_kv_heads, cols = min(SC, G - cg * SC);
  const int h0 = hk * G + cg * SC;                 // query head of column 0
  const int64_t qat = ((int64_t)st.k * H + h0) * HD;
  const int32_t* pages = c.table + (int64_t)st.seq * c.max_pages;
  const int64_t rowc = (int64_t)c.n_kv_heads * HD;
  char* rows = s_rows[wave];
  const char* kbase = (const char*)c.k + hk * HD * ESZ;
  const char* vbase = (const char*)c.v + hk * HD * ESZ;

  bf16x8_t qf[DS];     // the B operand
#pragma unroll
  for (int s = 0; s < DS; ++s)
    qf[s] = __builtin_bit_cast(
        bf16x8_t, c16 < cols ? *reinterpret_cast<const uint4*>(q + qat + c16 * HD + s * 32 + g * 8)
                             : make_uint4(0, 0, 0, 0));
  f32x4_t o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // of the weights' second parts, where V can be infinite (no e4m3 value is): their
  // product with it may be NaN or the other infinity, and must not meet the first's
  constexpr int DB2 = FP8 ? 1 : DB;
  f32x4_t o2[DB2];
#pragma unroll
  for (int i = 0; i < DB2; ++i) o2[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m_ref = -INFINITY, l_run = 0.0f;

  const int nblk = (st.t1 - st.t0 + kStepUnit - 1) / kStepUnit;   // blocks of each wave
  // keys of block i, one per lane (the upper half of the wave again), the pages
  // of block i + 1 read while block i's rows are on their way
  auto key_of = [&](int i) { return st.t0 + (i * 4 + wave) * SK + (lane & 31); };
  auto page_of = [&](int i) { return pages[min(key_of(i), st.t1 - 1) >> c.shift]; };
  auto slots_of = [&](int i, int page) { return c.slot(page, key_of(i), key_of(i) < st.t1); };
  u32x4_t kr[RI], vr[RI];
  uint8_t ksc[RI], vsc[RI];     // scale bytes
  // a key that is not there: slot 0 is read in its place, its score masked and
  // its V row cleared, the scale with it (slot 0's may be no number)
  auto fetch = [&](int sl) {
    const int sc = max(sl, 0);
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      const int s = __shfl(sc, i * RPI + lane / NCH, 64);
      const int64_t at = s * rowc * ESZ + lane % NCH * 16;
      // read once (by this entry)
      kr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(kbase + at));
      vr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(vbase + at));
      if constexpr (FP8) {
        ksc[i] = c.k_scale[(int64_t)s * c.n_kv_heads + hk];
        vsc[i] = c.v_scale[(int64_t)s * c.n_kv_heads + hk];
      }
    }
  };
  auto fk = [](int r) { return HD == 128 ? (r & 15) : ((r >> 1) & 7); };
  auto fv = [](int r) { return HD == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); };
  auto wide = [](uint32_t a, uint32_t b, uint8_t byte) {    // 8 codes to 8 bf16
    const float sc = scale_of(byte);
    return u32x4_t{fp8x2_to_bf16x2<false>(a, sc), fp8x2_to_bf16x2<true>(a, sc),
                   fp8x2_to_bf16x2<false>(b, sc), fp8x2_to_bf16x2<true>(b, sc)};
  };

  int page = 0;
  uint32_t there = 0;
  if (nblk > 0) {
    const int sl = slots_of(0, page_of(0));
    there = (uint32_t)__ballot(sl >= 0);
    page = page_of(1);
    fetch(sl);
  }
  for (int i = 0; i < nblk; ++i) {
    const uint32_t mask = there;
    // rows into LDS, chunk c of row r at c ^ f(r)
    auto put = [&](const u32x4_t (&x)[RI], const uint8_t (&sc)[RI], auto f) {
#pragma unroll
      for (int j = 0; j < RI; ++j) {
        const int r = j * RPI + lane / NCH, ch = lane % NCH;
        char* row = rows + r * ROWB;
        if constexpr (FP8) {
          *reinterpret_cast<u32x4_t*>(row + ((2 * ch) ^ f(r)) * 16) = wide(x[j][0], x[j][1], sc[j]);
          *reinterpret_cast<u32x4_t*>(row + ((2 * ch + 1) ^ f(r)) * 16) = wide(x[j][2], x[j][3], sc[j]);
        } else {
          *reinterpret_cast<u32x4_t*>(row + (ch ^ f(r)) * 16) = x[j];
        }
      }
    };
    put(kr, ksc, fk);
    wave_lds_order();
    f32x4_t s[2];
#pragma unroll
    for (int sb = 0; sb < 2; ++sb) {
      s[sb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const int r = sb * 16 + c16;
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) {
        const bf16x8_t a =
            *reinterpret_cast<const bf16x8_t*>(rows + r * ROWB + ((4 * ds + g) ^ fk(r)) * 16);
        s[sb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[ds], s[sb], 0, 0, 0);
      }
    }
    if (mask != ~0u)
#pragma unroll
      for (int j = 0; j < RI; ++j)
        if (!((mask >> (j * RPI + lane / NCH)) & 1)) {
          vr[j] = u32x4_t{0, 0, 0, 0};
          if constexpr (FP8) vsc[j] = kScaleOne;
        }
    wave_lds_order();
    put(vr, vsc, fv);      // over K
    wave_lds_order();
    if (i + 1 < nblk) {
      const int sl = slots_of(i + 1, page);
      there = (uint32_t)__ballot(sl >= 0);
      page = page_of(i + 2);
      fetch(sl);
    }
    if (mask != ~0u) {       // keys that are not there, or behind the stretch
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          s[sb][v] = (mask >> (sb * 16 + 4 * g + v)) & 1 ? s[sb][v] : -INFINITY;
    }
    float mb = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int v = 1; v < 4; ++v) mb = max3_raw(mb, s[0][v], s[1][v]);
    mb = max_column(mb) * scale_log2;
    if (__any(mb > m_ref + kLazy)) {
      const float mn = fmaxf(m_ref, mb);
      const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_ref - mn);
      m_ref = mn;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          o[d][v] *= alpha;
          if constexpr (!FP8) o2[d][v] *= alpha;
        }
    }
    const float msub = m_ref == -INFINITY ? 0.0f : m_ref;
    // A weight is the sum of two bf16 values, 16 bits of it, and the normaliser takes it
    // whole: the products wait for the keys, so a second one costs nothing (64 x 4096
    // 654 us with one and with two, in 8 bits 355 and 353; against 64 bits 0.0016 of the
    // result, its own rounding, and 0.0017).
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float a = s[y >> 1][2 * (y & 1)], b = s[y >> 1][2 * (y & 1) + 1];
      const float pa = __builtin_amdgcn_exp2f(fmaf(a, scale_log2, -msub));
      const float pb = __builtin_amdgcn_exp2f(fmaf(b, scale_log2, -msub));
      hi[y] = pack_bf16x2(pa, pb);
      lo[y] = pack_bf16x2(pa - __uint_as_float(hi[y] << 16),
                          pb - __uint_as_float(hi[y] & 0xffff0000u));
      l_run += pa + pb;
    }
    const bf16x8_t ph = __builtin_bit_cast(bf16x8_t, make_uint4(hi[0], hi[1], hi[2], hi[3]));
    const bf16x8_t pl = __builtin_bit_cast(bf16x8_t, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      s16x4 half[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int r = 16 * y + 4 * g + (c16 >> 2);
        const int ch = 2 * db + ((c16 & 3) >> 1);
        half[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(rows + r * ROWB + ((ch ^ fv(r)) * 16) + 8 * (c16 & 1)));
      }
      const bf16x8_t a = __builtin_bit_cast(
          bf16x8_t, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
      o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, ph, o[db], 0, 0, 0);
      f32x4_t& second = FP8 ? o[db] : o2[FP8 ? 0 : db];
      second = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pl, second, 0, 0, 0);
    }
    wave_lds_order();      // the next block's K, or the results, lie over V
  }

  if constexpr (!FP8)
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int v = 0; v < 4; ++v) o[d][v] += finite(o2[d][v]) ? o2[d][v] : 0.0f;

  // the four waves' results
  float l = l_run;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  float* so = (float*)rows;       // [SC][HD]: a wave's V rows hold SK * HD bf16
  static_assert(SC * HD * 4 <= SK * ROWB, "a wave's output fits its V rows");
  if (c16 < cols) {
    if (g == 0) {
      s_m[wave][c16] = m_ref;
      s_l[wave][c16] = l;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
      *reinterpret_cast<f32x4_t*>(so + c16 * HD + db * 16 + g * 4) = o[db];
  }
  __syncthreads();
  const bool whole = st.parts == 1;
  const int64_t at = ((int64_t)x * c.n_kv_heads + hk) * G + cg * SC;   // of the partial results
  for (int j = tid / (HD / 4); j < cols; j += 256 / (HD / 4)) {
    const int d = tid % (HD / 4) * 4;
    float m = s_m[0][j];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, s_m[w][j]);
    float ls = 0.0f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // a wave without keys has l = 0 and o = 0: its factor does not matter
      const float f = s_m[w][j] == m ? 1.0f : __builtin_amdgcn_exp2f(s_m[w][j] - m);
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>((const float*)s_rows[w] + j * HD + d);
      ls = fmaf(f, s_l[w][j], ls);
#pragma unroll
      for (int z = 0; z < 4; ++z) y[z] = fmaf(f, v[z], y[z]);
    }
    if (whole) {
      const float inv = ls == 0.0f ? 0.0f : 1.0f / ls;
      *reinterpret_cast<uint2*>(out + qat + j * HD + d) =
          make_uint2(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv));
    } else {
      float* pp = part + (at + j) * (HD + 4);
      *reinterpret_cast<float4*>(pp + 4 + d) = make_float4(y[0], y[1], y[2], y[3]);
      if (d == 0) *reinterpret_cast<float2*>(pp) = make_float2(m, ls);
    }
  }
  if (tid == 0 && st.part == 0 && hk == 0 && cg == 0) spans[st.k] = make_int2(x, st.parts);
}

// Joins the stretches of each entry that has several: a workgroup per (entry,
// head), whose groups of HD/4 threads (four dims a thread) take every PG-th stretch
// each and meet in LDS.  (One group for all stretches: 30 us for 126 of them.)
template <int HD>
__global__ __launch_bounds__(256) void paged_step_join_kernel(int H, Entries e,
                                                              const int2* __restrict__ spans,
                                                              const float* __restrict__ part,
                                                              bf16* __restrict__ out) {
  constexpr int PG = 256 / (HD / 4);
  __shared__ float s_m[PG], s_l[PG];
  __shared__ __attribute__((aligned(16))) float s_o[PG][HD];
  const int k = blockIdx.x, h = blockIdx.y, n = min(*e.n_active, e.max_active);
  if (k >= n) return;
  const int2 sp = spans[k];
  if (sp.y <= 1) return;
  const int pg = threadIdx.x / (HD / 4), d = threadIdx.x % (HD / 4) * 4;
  const int64_t step = (int64_t)H * (HD + 4);
  const float* pp = part + ((int64_t)sp.x * H + h) * (HD + 4);
  float m = -INFINITY, l = 0.0f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;
  for (int p0 = pg; p0 < sp.y; p0 += U * PG) {
    float2 ml[U];
    f32x4_t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* x = pp + min(p0 + u * PG, sp.y - 1) * step;
      ml[u] = *reinterpret_cast<const float2*>(x);
      v[u] = *reinterpret_cast<const f32x4_t*>(x + 4 + d);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p0 + u * PG >= sp.y) break;
      join(m, l, o, ml[u].x, ml[u].y, v[u]);
    }
  }
  if (d == 0) {
    s_m[pg] = m;
    s_l[pg] = l;
  }
  *reinterpret_cast<f32x4_t*>(&s_o[pg][d]) = o;
  __syncthreads();
  if (pg != 0) return;
  for (int x = 1; x < PG; ++x)
    join(m, l, o, s_m[x], s_l[x], *reinterpret_cast<const f32x4_t*>(&s_o[x][d]));
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  store4(out + ((int64_t)k * H + h) * HD + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
}

// want: stretches of the call's keys for each (K/V head, column group); least:
// units of a stretch at least
constexpr int64_t kMaxItems = (1 << 23) - 8;   // workgroups (their threads fit 32 bits)
struct StepShape {
  int groups, want, least, items;
  bool cut;          // whether an entry can have several stretches
  size_t off_part, bytes;
};
StepShape step_shape(const adept_paged_kv& kv, int n_heads, int max_active, int max_pages) {
  StepShape t{};
  const int G = n_heads / kv.n_kv_heads;
  t.groups = ceil_div(G, SC);
  const int64_t keys = (int64_t)max_pages * kv.page_size;
  t.want = std::max(1, kStepItems / (kv.n_kv_heads * t.groups));
  // A stretch has at least so many units.  Four where the entries alone fill the
  // card (64 sequences of up to 300 keys, 8 K/V heads: 15 us, 27 with one), two
  // where single units would be over 512 workgroups (16 of 1000: 19 us, 23; one of
  // 16000: 16 us, 22), else one (one of 700, 32 heads: 10 us, 12 with two).
  const int64_t base = (int64_t)max_active * kv.n_kv_heads * t.groups;
  t.least = base >= 256 ? 4 : base * ceil_div(keys, kStepUnit) > 512 ? 2 : 1;
  t.cut = keys > t.least * kStepUnit;
  const int64_t most = std::max<int64_t>(1, ceil_div(keys, t.least * kStepUnit));
  t.items = (int)std::min<int64_t>((int64_t)max_active + t.want, max_active * most);
  t.off_part = ((size_t)max_active * sizeof(int2) + 255) & ~(size_t)255;
  t.bytes = t.off_part;
  // fewer entries have shorter stretches: space also where only a smaller call cuts
  if (keys > kStepUnit)
    t.bytes += ((size_t)std::min(max_active, kStepEntries) + t.want) * n_heads *
               (kv.head_dim + 4) * sizeof(float);
  t.bytes = std::max<size_t>(t.bytes, 256);
  return t;
}
}  // namespace
}  // namespace adept

using namespace adept;

extern "C" size_t adept_paged_attend_workspace_bytes(const adept_paged_kv* kv, int n_heads,
                                                     int max_active, int n_seq, int max_pages) {
  if (!kv || kv->n_kv_heads <= 0 || n_heads < kv->n_kv_heads || max_active < 0 || n_seq <= 0 ||
      max_pages <= 0)
    return 256;
  return std::max(std::max(tile_shape(ADEPT_F32, *kv, n_heads, max_active, n_seq, max_pages).bytes,
                           tile_shape(ADEPT_BF16, *kv, n_heads, max_active, n_seq, max_pages).bytes),
                  step_shape(*kv, n_heads, max_active, max_pages).bytes);
}

namespace adept {

adept_status paged_attend_dispatch(adept_dtype dt, const adept_paged_kv* kv, int n_heads, float scale,
                                   int causal, const void* q, const int32_t* rows,
                                   const int32_t* n_active, int max_active, const int32_t* pos,
                                   const int32_t* seq, int n_seq, const int32_t* page_table,
                                   int max_pages, const int32_t* key_len, const uint8_t* key_live,
                                   void* out, void* workspace, size_t workspace_bytes,
                                   PagedKernels kernels, hipStream_t s) {
  ADEPT_TRY(paged_check("paged_attend", dt, kv));
  const int hd = kv->head_dim;
  ADEPT_REQUIRE(n_heads > 0 && n_heads <= 4096 && n_heads % kv->n_kv_heads == 0,
                "paged_attend: %d heads are no multiple of %d", n_heads, kv->n_kv_heads);
  ADEPT_REQUIRE(max_active >= 0 && max_active <= kMaxEntries && n_seq > 0 && max_pages > 0 &&
                    (int64_t)max_pages * kv->page_size <= kMaxTokens,
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
  const bool fp8 = kv->dtype == ADEPT_KV_FP8;
  if (dt == ADEPT_BF16 && tiles_fit(*kv) &&
      (kernels == kPagedAny ? max_active <= n_seq : kernels == kPagedSteps)) {
    const StepShape ss = step_shape(*kv, n_heads, max_active, max_pages);
    int2* spans = (int2*)workspace;
    float* part = (float*)((char*)workspace + ss.off_part);
    const int64_t items = (int64_t)ss.items * kv->n_kv_heads * ss.groups;
    ADEPT_REQUIRE(items <= kMaxItems, "paged_attend: too many entries");
#define ADEPT_STEP(HD, FP8)                                                                       \
  ADEPT_LAUNCH((paged_step_kernel<HD, FP8>), dim3((unsigned)items), dim3(256), 0, s, n_heads,     \
               ss.groups, ss.want, ss.least, sl, (const bf16*)q, e, c, (bf16*)out, spans, part)
    if (hd == 128) {
      if (fp8) ADEPT_STEP(128, true); else ADEPT_STEP(128, false);
    } else {
      if (fp8) ADEPT_STEP(64, true); else ADEPT_STEP(64, false);
    }
#undef ADEPT_STEP
    ADEPT_CHECK_LAUNCH("paged_step");
    if (ss.cut) {
      const dim3 jg(max_active, n_heads);
      if (hd == 128)
        ADEPT_LAUNCH(paged_step_join_kernel<128>, jg, dim3(256), 0, s, n_heads, e, spans, part,
                     (bf16*)out);
      else
        ADEPT_LAUNCH(paged_step_join_kernel<64>, jg, dim3(256), 0, s, n_heads, e, spans, part,
                     (bf16*)out);
    }
    return launch_status("paged_attend");
  }
  if (tiles_fit(*kv)) {
    const TileShape ts = tile_shape(dt, *kv, n_heads, max_active, n_seq, max_pages);
    char* w = (char*)workspace;
    int32_t* n_tiles = (int32_t*)w;
    Tile* tiles = (Tile*)(w + ts.off_tiles);
    float* part = (float*)(w + ts.off_part);
    const int64_t items = (int64_t)ts.max_tiles * kv->n_kv_heads * ts.parts;
    ADEPT_REQUIRE(items <= kMaxItems, "paged_attend: too many entries");
    ADEPT_LAUNCH(paged_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, e,
                 n_heads / kv->n_kv_heads, ts.max_tiles, (int32_t*)(w + ts.off_starts), tiles,
                 n_tiles);
    ADEPT_CHECK_LAUNCH("paged_plan");
    const dim3 grid((unsigned)((items + 7) / 8 * 8));
#define ADEPT_TILE(KERNEL, T, HD, FP8, THREADS)                                                  \
  ADEPT_LAUNCH((KERNEL<HD, FP8>), grid, dim3(THREADS), 0, s, n_heads, sl, (const T*)q, e, c,     \
               tiles, n_tiles, ts.max_tiles, ts.parts, (T*)out, part)
#define ADEPT_TILES(KERNEL, T, THREADS)                                                          \
  do {                                                                                           \
    if (hd == 128) {                                                                             \
      if (fp8) ADEPT_TILE(KERNEL, T, 128, true, THREADS);                                        \
      else ADEPT_TILE(KERNEL, T, 128, false, THREADS);                                           \
    } else {                                                                                     \
      if (fp8) ADEPT_TILE(KERNEL, T, 64, true, THREADS);                                         \
      else ADEPT_TILE(KERNEL, T, 64, false, THREADS);                                            \
    }                                                                                            \
  } while (0)
    if (dt == ADEPT_BF16) ADEPT_TILES(paged_tile_kernel, bf16, kTileThreads);
    else ADEPT_TILES(paged_tile_f32_kernel, float, kTile32Threads);
#undef ADEPT_TILES
#undef ADEPT_TILE
    ADEPT_CHECK_LAUNCH("paged_tile");
    if (ts.parts > 1) {
      const dim3 jg(ts.max_tiles, kv->n_kv_heads, TC_ * hd / 1024);
#define ADEPT_JOIN(T, HD)                                                                        \
  ADEPT_LAUNCH((paged_tile_join_kernel<T, HD>), jg, dim3(256), 0, s, n_heads, kv->n_kv_heads,    \
               tiles, n_tiles, ts.max_tiles, ts.parts, part, (T*)out)
      if (dt == ADEPT_BF16) {
        if (hd == 128) ADEPT_JOIN(bf16, 128); else ADEPT_JOIN(bf16, 64);
      } else {
        if (hd == 128) ADEPT_JOIN(float, 128); else ADEPT_JOIN(float, 64);
      }
#undef ADEPT_JOIN
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

}  // namespace adept

extern "C" adept_status adept_paged_attend(adept_dtype dt, const adept_paged_kv* kv, int n_heads,
                                           float scale, int causal, const void* q,
                                           const int32_t* rows, const int32_t* n_active,
                                           int max_active, const int32_t* pos, const int32_t* seq,
                                           int n_seq, const int32_t* page_table, int max_pages,
                                           const int32_t* key_len, const uint8_t* key_live,
                                           void* out, void* workspace, size_t workspace_bytes,
                                           void* stream) {
  return paged_attend_dispatch(dt, kv, n_heads, scale, causal, q, rows, n_active, max_active, pos,
                               seq, n_seq, page_table, max_pages, key_len, key_live, out, workspace,
                               workspace_bytes, kPagedAny, as_stream(stream));
}
