// bf16 GEMMs of at most 64 rows (decode, short prompts, the head of a few
// rows): one kernel, operands straight from global memory to the registers of
// v_mfma_f32_16x16x32_bf16, epilogue included.
//
// A workgroup of eight waves owns 16 or 32 weight rows (NB blocks of 16) and
// all M activation rows (MB blocks of 16).  Its waves take every eighth
// 64-deep (one cache line) piece of K; their f32 sums meet in LDS, in wave
// order, where the epilogue runs.  The weights cross HBM once, non-temporal;
// the activations (at most 64 rows) come from L2.  With the weights as the
// instruction's first operand a lane ends up with four consecutive output
// columns of one row, the unit the epilogues work on.
//
// What bounds these GEMMs is the weights' HBM time for wide layers and, for
// narrow ones, the chain of a kernel: its start, the row count, the row list,
// the operands, the hand-over of the sums.  So there is one kernel where a
// split over K with partial tiles in memory took two, the first weight loads
// are issued before the row count is known, and the row's RMSNorm factor and
// the row list of the fused decode schedule are formed on the way instead of
// by kernels of their own.  Measured, us, GEMM and epilogue kernel of the
// split form -> this one: 7B width, 1 row, a layer's four GEMMs with their
// norms and row list 131 -> 102 (4.5 TB/s of weights in gate/up); width 1600,
// 24 rows, QKV / first MLP 13.5 / 13.0 -> 11.0 / 10.3; width 768, 48 rows, biased
// QKV 9.4 -> 6.8, in the skinny path's order (SPLIT) 8.0.
#include <algorithm>
#include <cmath>

#include "gemm_tile.h"
#include "quant.h"

namespace adept {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
// in global memory: a pointer put together from two words is a flat one otherwise, whose
// loads go through the LDS counter too
typedef __attribute__((address_space(1))) u32x4_t global_u32x4_t;

// What the epilogue of one thread's four columns (n.. of row m) reads, loaded
// beside the first operands: each would be one more memory latency at the end.
struct DirPre {
  int m, n, row, slot;
  bool out;          // this lane stores (SwiGLU: the gate lanes)
  bf16x4_t bias, resid;
  float4 cs, sn;
  float sc;
};

// Four columns from n on of row m, any number of columns, any row stride.
__device__ __forceinline__ void store_any(const GP& p, int m, int n, const float (&v)[4]) {
  const int64_t at = (int64_t)m * p.ldc + n;
  const bool whole = n + 4 <= p.N;
  if (p.c_f32) {
    float* o = reinterpret_cast<float*>(p.C) + at;
    if (whole && ((uintptr_t)o & 15) == 0) {
      *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
      return;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (n + c < p.N) o[c] = v[c];
    return;
  }
  bf16* o = reinterpret_cast<bf16*>(p.C) + at;
  if (whole && ((uintptr_t)o & 7) == 0) {
    *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    return;
  }
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (n + c < p.N) o[c] = f2bf(v[c]);
}

// NB == 1 with a pair epilogue (rotary halves, gate and up): the 16 rows of the
// block are 8 of the first kind and their 8 partners.
//
// SPLIT: the sums in the order of the skinny path (gemm.hip), bit for bit: K in
// the segments its split sp gives these columns' tile, each one chain from zero,
// added up in ascending order.  The waves take every eighth segment.
//
// Q4: the weights in 4 bits (quant.h), in pieces of 128 of K: 16 bytes and four scale
// bytes of a lane are its operands of four products.  v_cvt_scalef32_pk_bf16_fp4 makes
// two bf16 of a byte, times the scale, exactly.  NB == 4 with a pair epilogue: two
// blocks of the first kind, then their partners.  A workgroup has 16 activation rows;
// those of the other rows of the same weights run on the same XCD, whose L2 then has
// them.  quant_form says which NB and W.
template <int EPI, int NB, int MB, int W, int U, bool SPLIT, bool Q4>
__global__ __launch_bounds__(64 * W) void gemm_direct_kernel(GP p, RowList rl, int row_norm,
                                                             SkSplit sp, QuantView qv) {
  static_assert(!(SPLIT && Q4) && (NB <= 2 || Q4) && (!Q4 || (MB == 1 && U == 1)), "forms");
  constexpr int KP = Q4 ? kQuantK : BK, HS = KP / 32;   // of K: a piece, products of one
  constexpr int HALF = NB == 4 ? 2 : 1;                 // blocks of one kind
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float4* red = reinterpret_cast<float4*>(smem);      // [wave or segment][MB * NB][64]
  __shared__ float ssq[W][MB * 16];
  __shared__ int32_t list[64];
  __shared__ uint8_t from2[64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  // Q4: the columns' workgroup and the first row
  int bx = blockIdx.x, m0 = 0;
  [[maybe_unused]] bool again = false;                  // the weights are read by others too
  if constexpr (Q4) {
    const int blocks = qv.row_blocks;
    if (blocks > 1) {
      const int i = bx >> 3;
      m0 = i % blocks * 16;
      bx = i / blocks * 8 + (bx & 7);
      if (bx >= qv.col_blocks) return;
      again = true;
    }
  }
  const int KT = Q4 ? (p.K + KP - 1) / KP : p.K / BK;
  const bool rope = EPI == EPI_QKV && p.rope_cos;
  const bool pair = EPI == EPI_SWIGLU || rope;
  // the first kind's first column, rows per kind, and the distance to the
  // second kind (SwiGLU's is in B2)
  const int per = pair && NB == 1 ? 8 : 16 * HALF;
  int n0, dn = 16;
  if (rope) {
    dn = p.head_dim >> 1;
    const int cpb = dn / per;   // blocks per head
    n0 = bx / cpb * p.head_dim + bx % cpb * per;
  } else {
    n0 = bx * (EPI == EPI_SWIGLU ? per : 16 * NB);
  }
  // raw list entries: loaded before the row count is known, used below it
  int raw[MB];
#pragma unroll
  for (int y = 0; y < MB; ++y)
    raw[y] = !rl.exit_layer && p.a_rows ? p.a_rows[min(m0 + 16 * y + r16, p.M_max - 1)]
                                        : m0 + 16 * y + r16;
  constexpr int XB = EPI == EPI_SWIGLU ? HALF : NB;
  constexpr int G = (MB * XB + W - 1) / W;            // epilogue groups of a wave
  DirPre pre[G];
  constexpr bool kRows = EPI == EPI_RESID || EPI == EPI_QKV;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const int t = wave + W * i, y = t / XB;
    pre[i].m = m0 + 16 * y + r16;
    pre[i].row = kRows && !rl.exit_layer ? p.rows[min(pre[i].m, p.M_max - 1)] : 0;
  }
  int el = INT_MAX, act = 0;
  if (rl.exit_layer) {
    if (lane < rl.n_tok) {
      el = rl.exit_layer[lane];
      act = rl.act[lane];
    }
  }
  // SPLIT: the segments of K, numbered from sp's first workgroup of the tile that
  // holds these columns
  [[maybe_unused]] const int u0 = SPLIT ? n0 / kSkinnyBN * KT : 0, w0 = SPLIT ? u0 / sp.U : 0;
  const int nseg = SPLIT ? (u0 + KT - 1) / sp.U - w0 + 1 : W;
  auto lo_of = [&](int s) { return max((w0 + s) * sp.U - u0, 0); };
  auto hi_of = [&](int s) { return min((w0 + s + 1) * sp.U - u0, KT); };
  const char* br[NB];
  [[maybe_unused]] const uint8_t* sr[NB];
  // Q4: a lane's place in a block of codes; the block is the wave's but where two kinds
  // share it, so that the loads have a scalar address
  constexpr bool kShared = NB == 1 && (EPI == EPI_SWIGLU || EPI == EPI_QKV);
  [[maybe_unused]] const uint32_t code_at = (uint32_t)(r16 * 16 + q * 256), scale_at = r16 * 4;
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    const bool second = pair && (NB == 1 ? r16 >= 8 : x >= HALF);   // a lane of the second kind
    const int r = NB == 1 ? (pair ? r16 & 7 : r16) : pair ? 16 * (x % HALF) + r16 : 16 * x + r16;
    const int row = n0 + r + (second && EPI != EPI_SWIGLU ? dn : 0);
    const bool b2 = EPI == EPI_SWIGLU && second;
    if constexpr (Q4) {
      // a block of columns behind the last (plain stores): the last one's, not stored
      int at = row >> 4;
      if constexpr (!kShared)
        at = (n0 >> 4) + (NB > 1 && pair ? x % HALF + (second && EPI != EPI_SWIGLU ? dn >> 4 : 0) : x);
      const int64_t blk = (int64_t)min(at, (p.N - 1) >> 4) * KT;
      br[x] = (const char*)(b2 ? qv.codes2 : qv.codes) + blk * kQuantBlock;
      sr[x] = (b2 ? qv.scales2 : qv.scales) + blk * kQuantScales;
      if constexpr (kShared) {   // the row of the block that the lane has is not r16
        br[x] += ((row & 15) - r16) * 16;
        sr[x] += ((row & 15) - r16) * 4;
      }
    } else {
      br[x] = (const char*)((b2 ? p.B2 : p.B) + (int64_t)row * p.ldb + 8 * q);
    }
  }
  constexpr int BH = Q4 ? 1 : HS;                       // loads of a weight piece
  u32x4_t bw[2][U][NB][BH], aw[2][Q4 ? 1 : U][MB][HS];
  [[maybe_unused]] uint32_t sw[2][U][NB];
  // a stage: up to U pieces of K from c0 on, below hi
  constexpr int kStep = SPLIT ? 1 : W;
  auto load_b = [&](int c0, int hi, int st) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * kStep;
      if (c >= hi) continue;   // uniform over the wave
#pragma unroll
      for (int x = 0; x < NB; ++x) {
        if constexpr (Q4) {
          const u32x4_t* w = reinterpret_cast<const u32x4_t*>(br[x] + (int64_t)c * kQuantBlock + code_at);
          bw[st][u][x][0] = again ? *w : __builtin_nontemporal_load(w);
          sw[st][u][x] = *reinterpret_cast<const uint32_t*>(sr[x] + (int64_t)c * kQuantScales + scale_at);
        } else {
#pragma unroll
          for (int h = 0; h < HS; ++h)
            bw[st][u][x][h] = __builtin_nontemporal_load(
                reinterpret_cast<const u32x4_t*>(br[x] + 2 * ((int64_t)c * BK + 32 * h)));
        }
      }
    }
  };
  if constexpr (SPLIT) {
    if (wave < nseg) load_b(lo_of(wave), hi_of(wave), 0);
  } else {
    load_b(wave, KT, 0);
  }

  // the rows: active rows, then (row list) the rows that exited before the
  // layer, in one ballot of at most 64 token rows
  int M = p.M_dev ? min(*p.M_dev, rl.exit_layer ? rl.max_act : p.M_max) : p.M_max;
  if (rl.ticket && blockIdx.x == 0 && threadIdx.x < 2) rl.ticket[threadIdx.x] = 0ull;
  const bf16* ar[MB];
  if (rl.exit_layer) {
    const int na = M;
    const bool ex = el < rl.layer;
    const uint64_t gone = __ballot(ex);
    M = min(na + __popcll(gone), 64);
    if (wave == 0) {
      const int at = na + __popcll(gone & ((1ull << lane) - 1));
      if (lane < na) {
        list[lane] = act;
        from2[lane] = 0;
      }
      if (ex && at < 64) {
        list[at] = lane;
        from2[at] = (el & 1) != ((rl.layer - 1) & 1);
      }
    }
    __syncthreads();
    if (M <= m0) return;
#pragma unroll
    for (int y = 0; y < MB; ++y) {
      const int m = min(m0 + 16 * y + r16, M - 1);
      ar[y] = (from2[m] ? p.A2 : p.A) + (int64_t)list[m] * p.lda + 8 * q;
    }
#pragma unroll
    for (int i = 0; i < G; ++i) pre[i].row = list[min(pre[i].m, M - 1)];
  } else {
    if (M <= m0) return;
#pragma unroll
    for (int y = 0; y < MB; ++y) {
      // rows past the count: row 0, computed and never stored
      const int row = m0 + 16 * y + r16 < M ? raw[y] : 0;
      ar[y] = ((p.a_sel && (p.a_sel[row] & 1)) ? p.A2 : p.A) + (int64_t)row * p.lda + 8 * q;
    }
#pragma unroll
    for (int i = 0; i < G; ++i)
      if (pre[i].m >= M) pre[i].row = 0;
  }
  auto load_a = [&](int c0, int hi, int st) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * kStep;
      if (c >= hi) continue;
#pragma unroll
      for (int y = 0; y < MB; ++y)
        if (y == 0 || 16 * y < M) {   // (Q4: one block)
#pragma unroll
          for (int h = 0; h < HS; ++h) {
            aw[st][u][y][h] = *reinterpret_cast<const u32x4_t*>(ar[y] + (int64_t)c * KP + 32 * h);
          }
        }
    }
  };
  // Q4: the activations of a round of pieces (one for each wave) go through LDS, where a
  // wave brings 16 / W rows of them in 1 KiB loads: straight from global memory to the
  // operands, 64 bytes of 16 rows a load, 16 rows of 4096 x 11008 took 14.2 us, 9.3 so.
  constexpr int kSeg = W * 256, kXRow = kSeg + 16;      // bytes of a row in a round, in LDS
  constexpr int kRowsW = 16 / W < 1 ? 1 : 16 / W, kLoads = 4 / kRowsW < 1 ? 1 : 4 / kRowsW;
  [[maybe_unused]] u32x4_t xw[4];
  [[maybe_unused]] const char* xr[kRowsW];
  [[maybe_unused]] auto load_x = [&](int round) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = i / kLoads;
      const int at = round * kSeg + i % kLoads * 1024;
      // rows that are not there and K behind the last are zeros: the codes there are
      // too, but 0 times what memory holds might be NaN
      xw[i] = u32x4_t{0, 0, 0, 0};
      if (m0 + kRowsW * wave + j < M && lane * 16 < 2 * p.K - at)
        xw[i] = *reinterpret_cast<const global_u32x4_t*>((uintptr_t)xr[j] + at + (uint32_t)(lane * 16));
    }
  };
  [[maybe_unused]] auto store_x = [&](int buf) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x4_t*>(smem + (buf * 16 + kRowsW * wave + i / kLoads) * kXRow +
                                  i % kLoads * 1024 + lane * 16) = xw[i];
  };
  if constexpr (Q4) {
    // a lane's row pointer from the lane that has it
    const uint64_t own = (uint64_t)(uintptr_t)(ar[0] - 8 * q);
#pragma unroll
    for (int j = 0; j < kRowsW; ++j) {
      const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)own, kRowsW * wave + j);
      const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(own >> 32), kRowsW * wave + j);
      xr[j] = (const char*)(uintptr_t)((uint64_t)hi << 32 | lo);
    }
    load_x(0);
  }
  if constexpr (SPLIT) {
    if (wave < nseg) load_a(lo_of(wave), hi_of(wave), 0);
  } else if constexpr (!Q4) {
    load_a(wave, KT, 0);
  }
  // the epilogue's inputs
#pragma unroll
  for (int i = 0; i < G; ++i) {
    DirPre& e = pre[i];
    const int t = wave + W * i, x = t % XB;
    const int kind = per == 8 ? q >> 1 : x / HALF;    // of a pair
    e.out = t < MB * XB && e.m < M && !(EPI == EPI_SWIGLU && per == 8 && kind);
    e.n = n0 + (per == 8 ? (EPI == EPI_SWIGLU ? 0 : kind * dn) + 4 * (q & 1)
                         : (HALF == 1 ? x * dn
                            : rope     ? kind * dn + 16 * (x % HALF)
                                       : 16 * x) + 4 * q);
    e.sc = 1.0f;
    e.bias = bf16x4_t{0, 0, 0, 0};
    if (!e.out) continue;
    if (p.row_scale) e.sc = p.row_scale[e.m];
    if (p.bias && Q4 && EPI == EPI_STORE) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (e.n + c < p.N) e.bias[c] = p.bias[e.n + c];
    } else if (p.bias) {
      e.bias = *reinterpret_cast<const bf16x4_t*>(p.bias + e.n);
    }
    if constexpr (EPI == EPI_RESID)
      e.resid = *reinterpret_cast<const bf16x4_t*>(p.resid + (int64_t)e.row * p.ldc + e.n);
    if constexpr (EPI == EPI_QKV) {
      e.slot = p.slot ? p.slot[e.row] : e.row;
      if (rope) {
        const int64_t o = (int64_t)p.pos[e.row] * dn + (e.n & (dn - 1));
        e.cs = rope4(p.rope_cos + o);
        e.sn = rope4(p.rope_sin + o);
      }
    }
  }
  f32x4_t acc[MB][NB];
  float ss[MB];
#pragma unroll
  for (int y = 0; y < MB; ++y) {
    ss[y] = 0.0f;
#pragma unroll
    for (int x = 0; x < NB; ++x) acc[y][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  auto step = [&](int c0, int hi, int st) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (c0 + u * kStep >= hi) continue;
#pragma unroll
      for (int h = 0; h < HS; ++h) {
        bf16x8_t bv[NB];
#pragma unroll
        for (int x = 0; x < NB; ++x) {
          if constexpr (Q4)
            bv[x] = quant_expand(bw[st][u][x][0][h], sw[st][u][x] >> (8 * h));
          else
            bv[x] = __builtin_bit_cast(bf16x8_t, bw[st][u][x][h]);
        }
#pragma unroll
        for (int y = 0; y < MB; ++y)
          if (y == 0 || 16 * y < M) {
            const u32x4_t a = aw[Q4 ? 0 : st][Q4 ? 0 : u][y][h];
#pragma unroll
            for (int x = 0; x < NB; ++x)
              acc[y][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  bv[x], __builtin_bit_cast(bf16x8_t, a), acc[y][x], 0, 0, 0);
            if (row_norm) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float lo = __uint_as_float(a[e] << 16);
                const float hi = __uint_as_float(a[e] & 0xffff0000u);
                ss[y] = fmaf(lo, lo, ss[y]);
                ss[y] = fmaf(hi, hi, ss[y]);
              }
            }
          }
      }
    }
  };
  auto hand_over = [&](int s) {   // the sums of segment s
#pragma unroll
    for (int y = 0; y < MB; ++y)
#pragma unroll
      for (int x = 0; x < NB; ++x)
        red[(s * MB * NB + y * NB + x) * 64 + lane] =
            make_float4(acc[y][x][0], acc[y][x][1], acc[y][x][2], acc[y][x][3]);
  };
  if constexpr (SPLIT) {
    // stage (s, c): pieces c.. of segment s; the next one may open the wave's
    // next segment, whose loads then pass the hand-over
    auto next = [&](int& s, int& c) {
      c += U;
      if (c >= hi_of(s)) {
        s += W;
        c = lo_of(s);
      }
    };
    auto finish = [&](int s) {
      hand_over(s);
#pragma unroll
      for (int y = 0; y < MB; ++y)
#pragma unroll
        for (int x = 0; x < NB; ++x) acc[y][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    };
    int s = wave, c = lo_of(wave);
#pragma unroll 1
    while (s < nseg) {
      int s1 = s, c1 = c;
      next(s1, c1);
      if (s1 < nseg) {
        load_b(c1, hi_of(s1), 1);
        load_a(c1, hi_of(s1), 1);
      }
      step(c, hi_of(s), 0);
      if (s1 != s) finish(s);
      s = s1;
      c = c1;
      if (s >= nseg) break;
      next(s1, c1);
      if (s1 < nseg) {
        load_b(c1, hi_of(s1), 0);
        load_a(c1, hi_of(s1), 0);
      }
      step(c, hi_of(s), 1);
      if (s1 != s) finish(s);
      s = s1;
      c = c1;
    }
  } else if constexpr (Q4) {
    const int rounds = (KT + W - 1) / W;
    auto piece = [&](int round, int st) {
      if (round * W + wave >= KT) return;
      const char* xb = smem + ((round & 1) * 16 + r16) * kXRow + wave * 256 + q * 16;
#pragma unroll
      for (int h = 0; h < HS; ++h) aw[0][0][0][h] = *reinterpret_cast<const u32x4_t*>(xb + 64 * h);
      step(round * W + wave, KT, st);
    };
    store_x(0);
#pragma unroll 1
    for (int r = 0; r < rounds; r += 2) {
      if (r + 1 < rounds) {
        load_x(r + 1);
        load_b((r + 1) * W + wave, KT, 1);
      }
      __syncthreads();
      piece(r, 0);
      if (r + 1 < rounds) {
        store_x(1);
        if (r + 2 < rounds) {
          load_x(r + 2);
          load_b((r + 2) * W + wave, KT, 0);
        }
        __syncthreads();
        piece(r + 1, 1);
        if (r + 2 < rounds) store_x(0);
      }
    }
    __syncthreads();   // the sums take the activations' place
    hand_over(wave);
  } else {
    const int mine = KT > wave ? (KT - wave + W - 1) / W : 0;   // this wave's pieces of K
    const int iters = (mine + U - 1) / U;
    auto at = [&](int it) { return it * U * W + wave; };
#pragma unroll 1
    for (int it = 0; it < iters; it += 2) {
      if (it + 1 < iters) {
        load_b(at(it + 1), KT, 1);
        load_a(at(it + 1), KT, 1);
      }
      step(at(it), KT, 0);
      if (it + 1 < iters) {
        if (it + 2 < iters) {
          load_b(at(it + 2), KT, 0);
          load_a(at(it + 2), KT, 0);
        }
        step(at(it + 1), KT, 1);
      }
    }
    hand_over(wave);   // a wave without pieces: zeros
  }
  if (row_norm) {
#pragma unroll
    for (int y = 0; y < MB; ++y) {
      float s = ss[y];
      s += __shfl_xor(s, 16, 64);
      s += __shfl_xor(s, 32, 64);
      if (q == 0) ssq[wave][16 * y + r16] = s;
    }
  }
  __syncthreads();
  // lane l of block (y, x): row 16 y + l % 16, four columns by l / 16
  auto sum = [&](int blk, int l) {
    float4 t = SPLIT ? make_float4(0.f, 0.f, 0.f, 0.f) : red[blk * 64 + l];
    auto add = [&](int w) {
      const float4 o = red[(w * MB * NB + blk) * 64 + l];
      t.x += o.x; t.y += o.y; t.z += o.z; t.w += o.w;
    };
    if constexpr (SPLIT) {
#pragma unroll 4
      for (int w = 0; w < nseg; ++w) add(w);
    } else {
#pragma unroll
      for (int w = 1; w < W; ++w) add(w);
    }
    return t;
  };
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const DirPre& e = pre[i];
    if (!e.out) continue;
    const int t = wave + W * i, y = t / XB, x = t % XB;
    float sc = e.sc;
    if (row_norm) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += ssq[w][e.m - m0];
      sc = 1.0f / sqrtf(s / (float)p.K + p.row_eps);
    }
    const float4 x4 = sum(y * NB + x, lane);
    const float bx[4] = {bf2f(e.bias[0]), bf2f(e.bias[1]), bf2f(e.bias[2]), bf2f(e.bias[3])};
    float v[4] = {x4.x * sc + bx[0], x4.y * sc + bx[1], x4.z * sc + bx[2], x4.w * sc + bx[3]};
    bf16x4_t o;
    if constexpr (EPI == EPI_STORE) {
      if constexpr (Q4) {
        store_any(p, e.m, e.n, v);
        continue;
      }
      if (p.c_f32) {
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(p.C) + (int64_t)e.m * p.ldc + e.n) =
            make_float4(v[0], v[1], v[2], v[3]);
        continue;
      }
    }
    bf16* dst = reinterpret_cast<bf16*>(p.C) + (int64_t)(EPI == EPI_RESID ? e.row : e.m) * p.ldc + e.n;
    if constexpr (EPI == EPI_SWIGLU) {
      const float4 y4 = per == 8 ? sum(y, lane ^ 32) : sum(y * NB + x + NB / 2, lane);
      const float u[4] = {y4.x * sc, y4.y * sc, y4.z * sc, y4.w * sc};
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = f2bf(silu(v[c]) * u[c]);
    } else if constexpr (EPI == EPI_QKV) {
      const int sec = e.n / p.d_q, cin = e.n - sec * p.d_q;
      dst = (sec == 0 ? p.q_out + (int64_t)e.m * p.d_q
                      : (sec == 2 ? p.v_cache : p.k_cache) + (int64_t)e.slot * p.d_q) + cin;
      if (rope && sec != 2) {
        const bool first = per == 8 ? q < 2 : x < HALF;
        const float4 y4 = per == 8 ? sum(y, lane ^ 32) : sum(y * NB + (x ^ (NB / 2)), lane);
        const float4 by = bias4(p.bias, first ? e.n + dn : e.n - dn);
        const float w[4] = {y4.x * sc + by.x, y4.y * sc + by.y, y4.z * sc + by.z, y4.w * sc + by.w};
        const float cv[4] = {e.cs.x, e.cs.y, e.cs.z, e.cs.w};
        const float sv[4] = {e.sn.x, e.sn.y, e.sn.z, e.sn.w};
#pragma unroll
        for (int c = 0; c < 4; ++c)
          o[c] = f2bf(first ? v[c] * cv[c] - w[c] * sv[c] : v[c] * cv[c] + w[c] * sv[c]);
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = f2bf(v[c]);
      }
    } else {
      if constexpr (EPI == EPI_GELU) gelu_erf(v);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        o[c] = f2bf(EPI == EPI_GELU_TANH   ? gelu_tanh(v[c])
                    : EPI == EPI_RESID     ? v[c] + bf2f(e.resid[c])
                                           : v[c]);
    }
    *reinterpret_cast<bf16x4_t*>(dst) = o;
  }
}

// LDS of a SPLIT workgroup's sums: at most this (beside the static arrays)
constexpr size_t kSplitLds = 128 * 1024;
// the most segments a tile has
int split_segments(const SkSplit& sp) {
  return sp.KT % sp.U == 0 ? sp.KT / sp.U : (sp.KT + sp.U - 2) / sp.U + 1;
}

template <int EPI, int NB, int MB, int W, int U, bool SPLIT, bool Q4 = false>
adept_status dir_launch(const GP& p, const RowList& rl, int row_norm, const char* name,
                        hipStream_t s, QuantView qv = QuantView{}) {
  SkSplit sp{};
  int parts = W;
  if (SPLIT) {
    sp = skinny_split(p.N, p.K);
    parts = split_segments(sp);
  }
  const size_t sums = (size_t)parts * MB * NB * 1024;
  const size_t red = Q4 ? std::max<size_t>(sums, 2 * 16 * (W * 256 + 16)) : sums;   // see kXRow
  static bool attr_set = false;
  if (SPLIT || red > 48 * 1024)
    ADEPT_TRY(lds_limit((const void*)gemm_direct_kernel<EPI, NB, MB, W, U, SPLIT, Q4>,
                        SPLIT ? kSplitLds : red, &attr_set, "gemm_direct LDS limit"));
  const int cols = EPI == EPI_SWIGLU ? 8 * NB : 16 * NB;
  int grid = ceil_div(p.N, cols);
  if (Q4) {
    qv.col_blocks = grid;
    qv.row_blocks = ceil_div(rl.exit_layer ? rl.n_tok : p.M_max, 16);
    if (qv.row_blocks > 1) grid = ceil_div(grid, 8) * 8 * qv.row_blocks;
  }
  {
    TimedLaunch tl(name ? name : "gemm_direct", s);
    hipLaunchKernelGGL((gemm_direct_kernel<EPI, NB, MB, W, U, SPLIT, Q4>), dim3(grid), dim3(64 * W), red,
                       s, p, rl, row_norm, sp, qv);
  }
  return launch_status("gemm_direct");
}

// 32 weight rows per workgroup where they still give half the chip one: the
// activations are read half as often (24 rows, width 1600: QKV 14.0 -> 11.0 us
// with 150 workgroups, but the O and down projections 12.4 -> 18.1 with 50)
bool dir_wide(int N, int epi) { return (epi == EPI_SWIGLU ? N / 16 : N / 32) >= 128; }

template <int EPI, bool SPLIT>
adept_status dir_rows(const GP& p, const RowList& rl, int row_norm, const char* name,
                      hipStream_t s) {
  const int M = rl.exit_layer ? rl.n_tok : p.M_max;
  // one piece of K in flight per stage for QKV, whose workgroups (768 of them at
  // the 7B width) are short and start with the row list: more of them per CU
  // (28 -> 24 us); two for the others (down and O projections 18 -> 15.6).
  // SPLIT: a wave's segment is four pieces at least and few waves have one (three
  // at K = 768), so its loads are issued together (twelve layers of width 768:
  // 12 rows 524 -> 500 us, 40 rows 687 -> 661)
  if (M <= 16)
    return dir_launch<EPI, 1, 1, 8, SPLIT ? 4 : EPI == EPI_QKV ? 1 : 2, SPLIT>(p, rl, row_norm, name,
                                                                               s);
  const bool wide = dir_wide(p.N, EPI);
  if (M <= 32)
    return wide ? dir_launch<EPI, 2, 2, 8, 2, SPLIT>(p, rl, row_norm, name, s)
                : dir_launch<EPI, 1, 2, 8, SPLIT ? 4 : 2, SPLIT>(p, rl, row_norm, name, s);
  return wide ? dir_launch<EPI, 2, 4, 8, 1, SPLIT>(p, rl, row_norm, name, s)
              : dir_launch<EPI, 1, 4, 8, SPLIT ? 2 : 1, SPLIT>(p, rl, row_norm, name, s);
}

// Weights in 4 bits: NB blocks of 16 weight rows, W waves.  The form with the least of
// an estimate of a CU's time, from its share of the workgroups: what their waves do a
// piece (the activations' part grows with the rows, the weights' with NB), their fixed
// part, and the rounds of pieces that wait for each other, of up to 16 waves at a time.
// The weights of the four were fitted to the times of 315 shapes (1 to 64 rows, n 320 ..
// 50304, k 512 .. 11008) before the loads had scalar addresses.  Of the kernel as it is,
// over the same shapes in all of NB = 1, 2, 4 and W = 4, 8, 16, the choice is 0.3 %
// behind the best of these five on average and 11 % at most, and 1.5 % and 17 % behind
// the best of all nine (64 rows of 8192 x 11008: 27.4 us with 4 x 4, 23.3 with 4 x 8).
// No form serves all, in graphs of 24 launches: 16 rows of 4096 x 11008 10.2 us with
// 1 x 16 and 15.1 with 4 x 16, 64 rows of 11008 x 4096 15.6 with 4 x 4 and 20.5 with
// 2 x 8, 1 row of 22016 x 4096 11.6 with 2 x 4 and 15.2 with 1 x 4.  More activation
// rows of a workgroup (32, 64) convert the weights less often, but few of them fit a
// CU: 64 rows of 11008 x 4096 18.6 us, where one block of them took 16.0.
struct QuantForm { int nb, w; };
QuantForm quant_form(int rows, int n_weights, int K) {
  static const QuantForm forms[] = {{1, 16}, {2, 16}, {2, 8}, {2, 4}, {4, 4}};
  const int pieces = ceil_div(K, kQuantK);
  QuantForm best{};
  double least = 0;
  for (const QuantForm& f : forms) {
    const double wgs = ceil_div((long)ceil_div(n_weights, 16 * f.nb) * ceil_div(rows, 16), 256);
    const int rounds = ceil_div(pieces, f.w);
    const double t = wgs * f.w * (rounds * (0.33 * std::min(rows, 16) / 16 + 1.6 * f.nb) + 2.6) +
                     20.0 * rounds * std::ceil(wgs * f.w / 16);
    if (best.nb == 0 || t < least) {
      best = f;
      least = t;
    }
  }
  return best;
}

template <int EPI>
adept_status quant_rows(const GP& p, const RowList& rl, int row_norm, const QuantView& qv,
                        const char* name, hipStream_t s) {
  const QuantForm f = quant_form(rl.exit_layer ? rl.n_tok : p.M_max,
                                 EPI == EPI_SWIGLU ? 2 * p.N : p.N, p.K);
  if (f.nb == 1) return dir_launch<EPI, 1, 1, 16, 1, false, true>(p, rl, row_norm, name, s, qv);
  if (f.nb == 2 && f.w == 16)
    return dir_launch<EPI, 2, 1, 16, 1, false, true>(p, rl, row_norm, name, s, qv);
  if (f.nb == 2 && f.w == 8)
    return dir_launch<EPI, 2, 1, 8, 1, false, true>(p, rl, row_norm, name, s, qv);
  if (f.nb == 2) return dir_launch<EPI, 2, 1, 4, 1, false, true>(p, rl, row_norm, name, s, qv);
  return dir_launch<EPI, 4, 1, 4, 1, false, true>(p, rl, row_norm, name, s, qv);
}

}  // namespace

// Up to 16 rows, or up to 64 of narrow layers.  With more rows each workgroup
// reads up to 64 activation rows for 16 or 32 weight rows, and the load path of
// the CUs binds: at the 7B widths and 64 rows 35 to 73 us a GEMM, 16 to 43 for
// the skinny path's two kernels; at width 1600 (10 M weights) a decode step of
// 24 rows 4000 us against 4530, of 40 4471 against 4661, of 48 the same, of 64
// 5412 against 5141; two layers of width 1600, 40 / 48 / 64 rows 152 / 162 / 185
// against 156 / 153 / 160.  Past 40 rows the line lies below the least width that
// lost (LayerNorm family, width 1024, 4.2 M: 48 / 64 rows 122 / 137 against 124 /
// 128), at the widest that was measured to win (width 768, 2.36 M: 108 / 118
// against 118 / 121); steps of the RMSNorm family would win up to 5.8 M (width 1024,
// 48 rows 103 against 127).  A step takes the form for all its GEMMs or none
// (layer.hip, encoder.hip).
// Plain stores (the head) of wide layers stream better through the tiles of
// gemm_mid.h (6 rows, 32000 x 4096: 52 us, 58 here).
bool gemm_direct_fits(int M_max, int n_weights, int K, int epi) {
  const int64_t weights = (int64_t)n_weights * K;
  const bool narrow = weights <= (M_max <= 40 ? 12 << 20 : 2400000);
  return M_max > 0 && M_max <= kDirectRows && epi != EPI_KV &&
         (narrow || (M_max <= 16 && epi != EPI_STORE));
}

bool gemm_direct_split_fits(int M_max, int N, int K, int epi) {
  if (epi == EPI_SWIGLU || !gemm_direct_fits(M_max, N, K, epi) || N % kSkinnyBN != 0) return false;
  const SkSplit sp = skinny_split(N, K);
  const int mb = M_max <= 16 ? 1 : M_max <= 32 ? 2 : 4, nb = M_max > 16 && dir_wide(N, epi) ? 2 : 1;
  return sp.G > 0 && (size_t)split_segments(sp) * mb * nb * 1024 <= kSplitLds;
}

bool gemm_direct_fits(const GemmArgs& g) {
  if (g.quant.codes) return g.M_max > 0 && (g.M_max <= kDirectRows || g.epi == EPI_STORE);
  if (g.few_rows == kFewSkinny) return false;
  if (g.few_rows == kFewSplit) return !g.rope_cos && gemm_direct_split_fits(g.M_max, g.N, g.K, g.epi);
  return gemm_direct_fits(g.M_max, g.epi == EPI_SWIGLU ? 2 * g.N : g.N, g.K, g.epi);
}

adept_status gemm_direct(const GemmArgs& g, hipStream_t s) {
  const GP p = to_gp(g);
  const RowList rl = g.list ? *g.list : RowList{};
  const int rn = g.row_norm ? 1 : 0;
  if (g.quant.codes) {
    switch (g.epi) {
      case EPI_STORE: return quant_rows<EPI_STORE>(p, rl, rn, g.quant, g.name, s);
      case EPI_QKV: return quant_rows<EPI_QKV>(p, rl, rn, g.quant, g.name, s);
      case EPI_RESID: return quant_rows<EPI_RESID>(p, rl, rn, g.quant, g.name, s);
      case EPI_SWIGLU: return quant_rows<EPI_SWIGLU>(p, rl, rn, g.quant, g.name, s);
      case EPI_GELU_TANH: return quant_rows<EPI_GELU_TANH>(p, rl, rn, g.quant, g.name, s);
      default: set_error("gemm: 4-bit weights without this epilogue"); return ADEPT_E_INVALID;
    }
  }
  if (g.few_rows == kFewSplit) {
    switch (g.epi) {
      case EPI_QKV: return dir_rows<EPI_QKV, true>(p, rl, rn, g.name, s);
      case EPI_RESID: return dir_rows<EPI_RESID, true>(p, rl, rn, g.name, s);
      case EPI_GELU: return dir_rows<EPI_GELU, true>(p, rl, rn, g.name, s);
      default: break;
    }
    set_error("gemm: few_rows = split without this epilogue");
    return ADEPT_E_INVALID;
  }
  switch (g.epi) {
    case EPI_STORE: return dir_rows<EPI_STORE, false>(p, rl, rn, g.name, s);
    case EPI_QKV: return dir_rows<EPI_QKV, false>(p, rl, rn, g.name, s);
    case EPI_RESID: return dir_rows<EPI_RESID, false>(p, rl, rn, g.name, s);
    case EPI_SWIGLU: return dir_rows<EPI_SWIGLU, false>(p, rl, rn, g.name, s);
    case EPI_GELU: return dir_rows<EPI_GELU, false>(p, rl, rn, g.name, s);
    case EPI_GELU_TANH: return dir_rows<EPI_GELU_TANH, false>(p, rl, rn, g.name, s);
    default: set_error("gemm: bad epilogue"); return ADEPT_E_INVALID;
  }
}

}  // namespace adept
