// Paged caches: what the store, the load and the attention share.
#pragma once

#include "common.h"

namespace adept {

// Scale bytes: 127 + E, -100 <= E <= 100.  Inside that range a code times its
// scale is a normal bf16 and f32 number and so is the scale's inverse.  A slot
// that was never written may hold any byte: 255 makes every code NaN, 0's too.
constexpr int kScaleMin = 127 - 100, kScaleMax = 127 + 100;
constexpr uint8_t kScaleOne = 127;
__device__ __forceinline__ float scale_of(uint8_t byte) { return __uint_as_float((uint32_t)byte << 23); }

// Two e4m3 codes (the low or the high half of w) times a power of two: exact
// in bf16 and in f32.
template <bool HI>
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
template <bool HI>
__device__ __forceinline__ float2 fp8x2_to_f32x2(uint32_t w, float scale) {
  const auto f = __builtin_amdgcn_cvt_pk_f32_fp8(w, HI);
  return make_float2(f[0] * scale, f[1] * scale);
}

// One layer's pages as a kernel sees them.
struct PagedView {
  const void *k, *v;
  const uint8_t *k_scale, *v_scale;
  const int32_t* table;   // [n_seq][max_pages]
  const uint8_t* live;    // by slot, nullable
  int max_pages, n_pages, shift, n_kv_heads, n_seq;
  // Slot of token t of a sequence from its page's number (-1: no key there).
  // Loops load the number a block ahead and ask for the slot when it is needed,
  // so that nothing waits for the load in between.
  __device__ __forceinline__ int slot(int page, int t, bool in) const {
    int s = in && (unsigned)page < (unsigned)n_pages ? (page << shift) | (t & ((1 << shift) - 1)) : -1;
    if (live) s = s >= 0 && live[s] ? s : -1;
    return s;
  }
};

// Which keys an entry sees: tokens 0 .. limit-1 of its sequence.
struct Entries {
  const int32_t *rows, *n_active, *pos, *seq, *key_len;
  int max_active, causal;
};
__device__ __forceinline__ int key_limit(const Entries& e, const PagedView& c, int seq, int pos) {
  if ((unsigned)seq >= (unsigned)c.n_seq) return 0;
  int n = c.max_pages << c.shift;
  if (e.causal) n = min(n, min(pos, INT_MAX - 1) + 1);
  if (e.key_len) n = min(n, e.key_len[seq]);
  return max(n, 0);
}
__device__ __forceinline__ int entry_limit(const Entries& e, const PagedView& c, int row, int* seq) {
  *seq = e.seq[row];
  return key_limit(e, c, *seq, e.causal ? e.pos[row] : 0);
}

constexpr int kMaxEntries = 1 << 23;   // rows or entries of a call (its grid's bound)
// slots of a cache and tokens of a sequence: a few blocks past them stay an int
constexpr int64_t kMaxTokens = INT_MAX - 1023;
inline int64_t paged_slots(const adept_paged_kv& kv) { return (int64_t)kv.n_pages * kv.page_size; }
// adept_paged_attend with the kernels named: those for one entry per sequence, for
// many, or (kPagedAny) by the counts
enum PagedKernels { kPagedAny = 0, kPagedSteps = 1, kPagedTiles = 2 };
adept_status paged_attend_dispatch(adept_dtype dt, const adept_paged_kv* kv, int n_heads, float scale,
                                   int causal, const void* q, const int32_t* rows,
                                   const int32_t* n_active, int max_active, const int32_t* pos,
                                   const int32_t* seq, int n_seq, const int32_t* page_table,
                                   int max_pages, const int32_t* key_len, const uint8_t* key_live,
                                   void* out, void* workspace, size_t workspace_bytes,
                                   PagedKernels kernels, hipStream_t s);
// the checks of a cache descriptor; `what` names the entry point
adept_status paged_check(const char* what, adept_dtype dt, const adept_paged_kv* kv);

}  // namespace adept
