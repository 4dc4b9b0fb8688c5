// What the calls that move rows between memory and a quantised cache share: how a
// wavefront finds the (sequence, block) that it works on and the block's rows, and the
// pieces of moving them.
#pragma once

#include "device_common.h"

namespace pa {
namespace dev {
namespace {

constexpr int kExpBias = 127;

struct KvRowArgs {
  const int32_t* bt;
  const int32_t* seq_lens;
  const int32_t* cu;
  uint8_t* kc;
  uint8_t* vc;
  uint8_t* scales;
  int64_t k_stride, v_stride;
  int32_t max_blocks, n_seqs, n_tokens, num_blocks, hkv;
  int64_t slots;    // (sequence, block) slots of the launch
  bool by_token;    // a slot per row, not per block
};

// One block of the launch and its rows.
struct BlockRows {
  int id;          // block, as the table has it
  int off0, off1;  // token offsets [off0, off1) of the block have rows; none: nothing to do
  int row0;        // row of offset off0
};

// Largest r of [0, n) with key(cu[r], r) <= x (keys rise with r): each round compares
// 64 evenly spaced sequences, one per lane.
template <class Key>
__device__ __forceinline__ int find_seq(const int32_t* cu, int n, int x, Key key) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + lane * step;
    const bool below = i < hi && key(cu[i < hi ? i : lo], i) <= x;
    const int c = max(1, __popcll(__ballot(below)));
    lo += (c - 1) * step;
    hi = min(lo + step, hi);
  }
  return lo;
}

__device__ __forceinline__ BlockRows find_rows(const KvRowArgs& a, int slot) {
  const BlockRows none{-1, 0, 0, 0};
  int r, c0, n, L;
  int64_t j;  // logical block
  if (a.by_token) {
    // row `slot` is a block's first one; a guess that is right in a decode step, where
    // every sequence has one row, saves the search
    r = min(slot, a.n_seqs - 1);
    if (a.cu[r] != slot || a.cu[r + 1] != slot + 1)
      r = find_seq(a.cu, a.n_seqs, slot, [](int c, int) { return c; });
    c0 = a.cu[r], n = a.cu[r + 1] - c0, L = a.seq_lens[r];
    const int row = slot - c0, pos = L - n + row;
    if (row < 0 || row >= n || pos < 0 || (row > 0 && pos % kBlock)) return none;
    j = pos / kBlock;
  } else {
    r = find_seq(a.cu, a.n_seqs, slot, [](int c, int i) { return c / kBlock + 2 * i; });
    c0 = a.cu[r], n = a.cu[r + 1] - c0, L = a.seq_lens[r];
    j = (L - n) / kBlock + (int64_t)slot - (c0 / kBlock + 2 * r);
  }
  const int first = L - n;  // first row's position
  if (n <= 0 || first < 0 || c0 < 0 || j < 0 || j * kBlock >= L || j >= a.max_blocks) return none;
  const int p0 = int(j) * kBlock, off0 = max(first - p0, 0);
  const int row0 = c0 + p0 + off0 - first;
  // cu may run past the caller's rows
  const int off1 = min(min(L - p0, kBlock), off0 + max(a.n_tokens - row0, 0));
  if (off1 <= off0) return none;
  return {a.bt[(int64_t)r * a.max_blocks + j], off0, off1, row0};
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Eight values of T as loaded, and as float32.  Non-temporal where a load takes whole lines:
// the rows are read once (64 bf16 prompts whose rows are in no cache 49 us, 55 with plain
// loads; 46 where the last-level cache holds them all).  A float32 row's lines are read in two
// halves of each lane's 32 bytes, the second from the cache (128000 tokens, 8 kv-heads of 128,
// to the 4-bit cache 243 us, 258 with non-temporal loads, to the 8-bit one 257 and 276).
template <typename T>
struct Raw8 {
  u32x4 x[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (size_t i = 0; i < sizeof(T) / 2; ++i) {
      const u32x4* q = reinterpret_cast<const u32x4*>(p + 16 / sizeof(T) * i);
      x[i] = sizeof(T) == 2 ? __builtin_nontemporal_load(q) : *q;
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 2) return __uint_as_float(i % 2 ? x[0][i / 2] & 0xFFFF0000u : x[0][i / 2] << 16);
    else return __uint_as_float(x[i / 4][i % 4]);
  }
};

// Transpose of 4 x 4 bytes: byte i of word k becomes byte k of word i.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
  w[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
  w[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
  w[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

// Slots of n rows of n_seqs sequences: one per row where that is fewer than two per
// sequence and one per 16 rows (decode and verification steps).
KvRowArgs with_slots(KvRowArgs a) {
  a.slots = int64_t(a.n_tokens) / kBlock + 2 * int64_t(a.n_seqs);
  a.by_token = a.n_tokens <= a.slots;
  if (a.by_token) a.slots = a.n_tokens;
  return a;
}

}  // namespace
}  // namespace dev
}  // namespace pa
