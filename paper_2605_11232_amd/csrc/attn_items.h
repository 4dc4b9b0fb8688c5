// bf16 paged attention over a prefix-shared KV cache on CDNA4 MFMA.
//
// What is computed (paper: Section 2, PagedAttention's block table and
// Automatic Prefix Caching; Section 3, cached shared prefixes give the result
// of recomputing them): for each query row, softmax(scale * q K^T) V over the
// keys 0..a of its sequence, where a is the query's logical position, keys
// and values gathered block by block through the block table.
//
// Item kinds of one launch (see plan.cpp):
//  * tile items, one workgroup of 4 wavefronts x 32 rows: 64-key steps of K
//    and V^T are copied from the paged cache straight into LDS (two stages)
//    and shared by the four wavefronts; S^T = K Q^T and O^T += V^T P^T run on
//    32x32x16 MFMA.  Computing the transposed score tile puts one query row
//    in each lane, so the online-softmax row max needs a single cross-lane
//    exchange, and the probabilities are already laid out as the B operand
//    of the PV product (no LDS round trip for P).
//  * shared-prefix items: the tile path over gathered rows of sequences whose
//    leading blocks coincide (cascade); partial results are merged.
//  * row items, one wavefront each: up to 32 rows (decode's G rows, or a
//    verification sequence's n_q * G rows cut in pieces) as one or two
//    16-column tiles of 16x16x32 MFMA, with K and V^T streamed straight from
//    HBM into registers over a split of the key range.
//
// The key order inside a tile is permuted so that each lane's eight PV
// k-elements are eight consecutive keys: then V^T operands are single 16-byte
// reads of the cache's [head_dim][block] value layout.
//
// The same items read the 8-bit cache (KV8): e4m3 values with a power-of-two
// scale per (block, kv-head) of keys and of values.  e4m3 holds four significant
// bits, so a value times its scale is a bf16 number: operands are converted
// exactly, and an item computes what it would over a bf16 cache of those numbers.
// And the 4-bit cache (KV4): e2m1 codes, for each token a power of two for 32 dims of
// its key and one for its value.  Keys become bf16 with their scales, as there; a value's
// scale multiplies the token's probability in float32 before that is rounded to bf16 (a
// power of two: no further rounding), so that the codes alone are the product's operand.
//
// Scores are scaled by scale * log2(e) and exponentiated with exp2; the
// natural-log LSE is recovered as ln2 * (m + log2 l).
#pragma once

#include <hip/hip_ext.h>

#include "device_common.h"
#include "plan_format.h"

namespace pa {
namespace dev {
// The compiler's name for v_mul_legacy_f32: zero times anything is zero.
__device__ float fmul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");

struct AttnArgs {
  const __bf16* q;
  const __bf16* kc;  // 8 and 4 bits: the caches' bytes
  const __bf16* vc;
  const int32_t* bt;
  const int32_t* seq_lens;
  const int32_t* cu_q;
  const int32_t* plan;
  __bf16* out;
  float* lse;
  float* ws_o;
  float* ws_lse;
  int32_t max_blocks;
  int32_t num_blocks;
  int32_t hq;
  int32_t hkv;
  int32_t group;
  int32_t merge_narrow;  // narrow merge-group templates, or -1: as the plan says
  float scale_log2;
  // 8 bits: [num_blocks][hkv][2], exponent + 127 of keys and of values; 4 bits:
  // [num_blocks][hkv][D/32 + 1][16]
  const uint8_t* scales;
};

namespace {

// Row r of a tile's K buffer holds key perm32(r): bits 2 and 3 swapped.
__device__ __forceinline__ int perm32(int r) {
  return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1);
}

// Tile items walk the keys in steps of kTileSub 32-key sub-tiles (2 kTileSub
// cache blocks).  Smaller steps halve the LDS and registers a workgroup holds,
// so more workgroups share a CU.
#ifndef PA_TILE_SUB
#define PA_TILE_SUB 2
#endif
constexpr int kTileSub = PA_TILE_SUB;
static_assert(kTileSub == 1 || kTileSub == 2, "32- or 64-key tile steps");
constexpr int kTileWavesPerEu = kTileSub == 1 ? 3 : 2;

// LDS of a tile item: K and V^T of two steps, each step held as the cache's
// own 2 NSUB blocks (the grouped key layout [D/32][16 slots][32] for K,
// [D][16 keys] for V^T).  Blocks are copied straight from global memory into
// LDS (no register staging), each 64-unit (1 KB) piece of LDS from one
// contiguous 1 KB of the cache; the 16-byte units are XOR-swizzled within a
// piece so that the MFMA operand reads of 16 consecutive lanes fall in
// distinct banks:
//  K:   block b, 32-dim group c, slot position s, 8-dim unit p
//         -> unit (b D/32 + c) 64 + 4 s + (p ^ (s / 4 % 4))
//  V^T: dim row d, half h (8 keys)         -> unit 2 d + (h ^ vswz(d))
// Slot position s of a block holds offset s with bits 2 and 3 swapped, so
// row r of a step's 32-key tile (position r % 16 of its block) holds key
// 32 * (r / 32) + perm32(r % 32).
template <int D, int NSUB, int BITS>
struct TileSmem {
  static constexpr int BLK = kBlock * D;  // bf16 per block of K or V^T
  __bf16 k[2][2 * NSUB * BLK];
  __bf16 v[2][2 * NSUB * BLK];
  float sv[2][BITS == 4 ? 32 * NSUB : 1];  // KV4: the values' scales of a step's tokens
};

__device__ __forceinline__ int vswz(int d) { return ((d >> 2) ^ (d >> 3)) & 1; }

// Cache-policy bits of a buffer load on gfx950: non-temporal.
constexpr int kCachePolicyNonTemporal = 2;

// s_waitcnt vmcnt(0): every global load of this wavefront, including the
// copies into LDS, has completed.
__device__ __forceinline__ void wait_vmem() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// Asynchronous copy of 16 bytes per lane into LDS: lane l reads bytes
// [off, off + 16) of the wave-uniform block `base` (a buffer resource in
// scalar registers, so the per-copy address work is scalar) and writes them
// to bytes [16 l, 16 l + 16) after `lds` (wave-uniform).  Offsets at or past
// `bytes` read zeros instead of faulting.
// STREAM: the non-temporal cache policy (data read once: the lines are not
// kept in L2 at the expense of data other items re-read).
template <bool STREAM = false>
__device__ __forceinline__ void copy16_to_lds(const void* base, int bytes, uint32_t off, __bf16* lds) {
  const __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, bytes, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, off, 0, 0,
                                           STREAM ? kCachePolicyNonTemporal : 0);
}

// Power of two of a scale byte (exponent + 127).
__device__ __forceinline__ float scale8(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four e4m3 values times a power of two, as bf16 (exact).
__device__ __forceinline__ u32x2 bf16_of_e4m3(uint32_t x, float scale) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true))};
}
__device__ __forceinline__ u32x4 bf16_of_e4m3(uint32_t x0, uint32_t x1, float scale) {
  const u32x2 a = bf16_of_e4m3(x0, scale), b = bf16_of_e4m3(x1, scale);
  return u32x4{a[0], a[1], b[0], b[1]};
}

// Eight e2m1 codes as bf16 (exact), times the power of two whose exponent bits `scale`
// has (all ones: NaN); its other bits do not count.
__device__ __forceinline__ u32x4 bf16_of_e2m1(uint32_t x, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3))};
}
// Byte i of a word where bf16_of_e2m1 looks for an exponent.
__device__ __forceinline__ float exponent_byte(uint32_t x, int i) {
  return __uint_as_float(i == 3 ? x >> 1 : x << (23 - 8 * i));
}
// p times a token's value scale: zero where p is, whatever the scale of a token that the
// row does not see; where it sees one whose scale stands for NaN, infinity, which a code of
// zero makes NaN.
__device__ __forceinline__ float times_scale(float p, float scale) {
  return fmul_legacy(p, scale);
}

// Sum of the eight bf16 values of a vector added to acc (v_dot2 with ones).
__device__ __forceinline__ float add_bf16x8(bf16x8 v, float acc) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    acc = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{v[2 * i], v[2 * i + 1]}, one, acc, false);
  return acc;
}

#ifndef PA_LDS_PREFETCH
#define PA_LDS_PREFETCH 3
#endif
// N MFMAs whose A operands are 16-byte LDS reads (addr(i) gives the address
// of MFMA i), with PF reads in flight ahead of the MFMA that uses them: LDS
// latency is hidden behind the MFMAs instead of being paid before each one.
// The scheduling-group barriers keep the read-ahead order in the code.
template <int N, int PF, class AddrF, class MfmaF>
__device__ __forceinline__ void lds_mfma_pipeline(AddrF addr, MfmaF mfma) {
  static_assert(PF >= 1 && PF <= N, "read-ahead depth");
  u32x4 x[PF];
#pragma unroll
  for (int i = 0; i < PF; ++i) x[i] = ld16(addr(i));
  __builtin_amdgcn_sched_group_barrier(0x100, PF, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const u32x4 a = x[i % PF];
    if (i + PF < N) {
      x[i % PF] = ld16(addr(i + PF));
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    mfma(i, a);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
  }
}

// max of a value over the two lane halves (lane l and l ^ 32)
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Tile item (SHARED = false): 128 rows of one sequence, causal.  Shared-prefix
// item (SHARED = true): 128 gathered rows of a cascade group's members over
// keys every one of them sees; results go to the members' partial rows.
//
// Software pipeline over steps, one workgroup barrier per step: the softmax of
// step t, then the score MFMAs of step t + 1 and the PV MFMAs of step t, beside
// the softmax of the SIMD's other wavefronts.  K of step t + 2 and V^T of step t + 1 are copied into the LDS
// buffers freed by steps t and t - 1 during step t.
//
// KV8: a step's K and V^T pass through registers, where they become bf16, into
// the same LDS tiles: step t stores K of step t + 2 and V^T of step t + 1, loaded
// during step t - 1, and loads the next.  Each value is converted once per
// workgroup, not once per wavefront that reads it: 32 prompts on 2048 cached tokens
// take 792 to 825 us on different cards, on one of them 811 against 741 over a bf16 cache
// of the same values; the conversions are 32 VALU instructions in about 160 a step, the
// float32 sums 16.
//
// KV4: the same stages; a wavefront loads block w of a step, D / 8 bytes of K and of V^T
// a lane (part of a token's key; a dim's 16 tokens, at head_dim 128 of two dims).
template <int D, int NSUB, int BITS, bool SHARED, bool FULL, bool STREAM = false>
__device__ __forceinline__ void tile_item(const int32_t* it, int g, int poff, const AttnArgs& a,
                                          TileSmem<D, NSUB, BITS>& sm) {
  constexpr bool KV8 = BITS == 8, KV4 = BITS == 4;
  constexpr bool STAGED = KV8 || KV4;
  constexpr int KT = 32 * NSUB;     // keys per step
  constexpr int NB = KT / kBlock;   // blocks per step
  constexpr int NI = NSUB * D / 64; // LDS copies per wavefront per step, for each of K and V^T
  constexpr int BLK = TileSmem<D, NSUB, BITS>::BLK;
  const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, hh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6) & 3;
  const int G = a.group;
  const int lr = w * 32 + j;
  const int row0 = it[I_ROW0], nrows = it[I_NROWS], kv0 = it[I_KV0];
  const bool valid = lr < nrows;
  int key_seq, kend, qs, qi, hq, apos, wg_amin, part;
  if constexpr (SHARED) {
    // gathered row -> member sequence and its own row
    const int rpm = it[S_RPM];
    const int rg = row0 + lr;
    const int mi = rg / rpm, rl = rg - mi * rpm;
    const int32_t* mem = a.plan + it[S_MEMBERS] + 2 * (valid ? mi : 0);
    const int seq = mem[0];
    qs = a.cu_q[seq];
    qi = rl / G;
    hq = g * G + (rl - qi * G);
    part = mem[1] + poff + rl;
    key_seq = it[S_BLOCK_SEQ];
    kend = it[S_KV1];
    apos = kend - 1;               // every shared key is visible
    wg_amin = kend - 1;            // only a partial last step is masked
  } else {
    const int r = it[I_SEQ];
    const int L = a.seq_lens[r];
    qs = a.cu_q[r];
    const int n = a.cu_q[r + 1] - qs;
    const int rho = row0 + lr;
    qi = rho / G;
    hq = g * G + (rho - qi * G);
    part = it[I_PART] < 0 ? -1 : it[I_PART] + poff + lr;
    key_seq = r;
    // the range may run past the last key that the item's last row sees
    kend = min(it[I_KV1], L - n + (row0 + nrows - 1) / G + 1);
    // Lanes without a row see every key (their scores are zero): seeing none they would
    // never have a reference, and the wavefront would look for one in each masked step.
    apos = valid ? L - n + qi : kend - 1;
    // Rows are ordered by query, so the item's first row has the smallest
    // position: steps entirely at or below it need no causal mask.
    wg_amin = L - n + row0 / G;
  }

  bf16x8 qf[D / 16];
  {
    const __bf16* qp = a.q + ((int64_t)(qs + qi) * a.hq + hq) * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = as_bf16x8(valid ? ld16(qp + 16 * ks) : zero16());
  }
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[dt][e] = 0.f;
  // Running reference max m (raw scores) and this lane's partial row sum l
  // (the two lane halves hold disjoint keys of the same row; they are added
  // at the end).  p = exp2(c * s - mc) with c = scale * log2(e), mc = c * m.
  const float c = a.scale_log2;
  float m = kNegInf, mc = 0.f, l = 0.f;

  // Per-lane byte offsets of this wavefront's LDS copies inside a block: copy
  // i fills LDS units 64 * (4 i + w) + lane of the step buffer.
  uint32_t koff[NI], voff[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int U = 64 * (4 * i + w) + lane;
    // K: LDS piece 4 i + w is 32-dim group (4 i + w) % (D/32) of a block
    const int grp = (4 * i + w) % (D / kKeyGroup), pos = lane >> 2;
    const int unit = (lane & 3) ^ ((pos >> 2) & 3);
    koff[i] = (uint32_t)((grp * kBlock * kKeyGroup + pos * kKeyGroup + 8 * unit) * 2);
    const int u = U % (2 * D), d = u >> 1, h = (u & 1) ^ vswz(d);
    voff[i] = (uint32_t)((d * kBlock + 8 * h) * 2);
  }
  const int32_t* bt = a.bt + (int64_t)key_seq * a.max_blocks;
  constexpr int kHeadBytes = kBlock * D * BITS / 8;  // one (block, kv-head) of K or V^T
  const char* kbase = reinterpret_cast<const char*>(a.kc) + (int64_t)g * kHeadBytes;
  const char* vbase = reinterpret_cast<const char*>(a.vc) + (int64_t)g * kHeadBytes;
  const int64_t blk_bytes = (int64_t)a.hkv * kHeadBytes;  // one block, all kv-heads

  // Block ids of a step (wave-uniform), clamped into the cache when the
  // window of 64 table entries is fetched.  Blocks at or past kend read the
  // item's last block again, so every copy reads inside the cache; their keys
  // are masked and their values zeroed before use.  Steps advance NB blocks
  // from the window's first block, so a step's blocks never straddle two
  // windows: one window check per step.
  BlockWindow win;
  win.init(bt, kend > 0 ? (kend - 1) / kBlock : 0, a.num_blocks, kv0 / kBlock);
  // blk[b]: byte offset of the step's block b (all kv-heads per block), so
  // each block's address is computed once for its K and its V^T copies
  auto step_blocks = [&](int t0, int64_t (&blk)[NB]) {
    const int jb = t0 / kBlock;
    win.seek(jb);
#pragma unroll
    for (int b = 0; b < NB; ++b)
      blk[b] = (int64_t)((uint64_t)(uint32_t)win.at(jb + b) * (uint32_t)blk_bytes);  // ids >= 0
  };
  // Copy slot i of wavefront w lands in block (4 i + w) * 64 / (2 D) of the
  // step: block i for D = 128, block 2 i + w / 2 for D = 64.
  static_assert(NI >= 1, "at least one copy per wavefront");
  static_assert(D == 64 || D == 128, "head_dim 64 or 128");
  auto copy_block = [&](const int64_t (&blk)[NB], int i) {
    if constexpr (D == 128) return blk[i];
    else return blk[2 * i] + ((w >> 1) & 1) * (blk[2 * i + 1] - blk[2 * i]);  // no indexed array
  };
  // STREAM items (keys no other item reads) copy with the non-temporal
  // policy, leaving L2 to the keys other items re-read (shared prefixes,
  // the other tiles of a long sequence).
  auto issue_k = [&](const int64_t (&blk)[NB], int buf) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      copy16_to_lds<STREAM>(kbase + copy_block(blk, i), kHeadBytes, koff[i],
                            &sm.k[buf][512 * (4 * i + w)]);
  };
  auto issue_v = [&](const int64_t (&blk)[NB], int buf) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      copy16_to_lds<STREAM>(vbase + copy_block(blk, i), kHeadBytes, voff[i],
                            &sm.v[buf][512 * (4 * i + w)]);
  };

  // KV8 staging: a wavefront loads 1 KB pieces, 16 bytes per lane: piece 4 i + w
  // of a step is 64 head dims of block (4 i + w) / (D / 64).  Of K a lane takes
  // 16 dims of one slot and writes two 16-byte units; eight neighbouring lanes
  // (four slots) write in distinct banks.  Of V^T it takes one dim's 16 keys.
  static_assert(!STAGED || NSUB == 2, "staging through registers: 64-key steps");
  constexpr int NR = KV8 ? NSUB * D / 128 : 1;
  u32x4 rk[NR], rv[NR];   // raw K and V^T on their way
  int64_t blk8[2][NR];    // byte offsets of the blocks of this wavefront's pieces, by step % 2
  uint32_t sc8[2][NR];    // their scales: keys' byte, values' byte
  const int slot8 = (lane >> 1) & 15, pos8 = key_slot_pos(slot8);
  const uint32_t piece_off = D == 128 ? (w & 1) * 1024 : 0;  // of a piece in its block
  const uint32_t koff8 = piece_off + slot8 * 64 + 32 * hh + 16 * (lane & 1);
  const uint32_t kdst8 = hh * 64 + 4 * pos8 + ((2 * (lane & 1)) ^ ((pos8 >> 2) & 3));
  // Blocks and scales of a step's pieces.  A block is 16 D hkv bytes, its scales are 2
  // hkv; a pair lies in one aligned word (the array's memory is whole words), which a
  // scalar load takes (16-bit vector loads: 32 prompts 816 us against 805, 256 decode
  // requests 77.6 against 75.7).
  auto step_blocks8 = [&](int t0, int s) {
    const int jb = t0 / kBlock;
    win.seek(jb);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const uint64_t id = (uint32_t)win.at(jb + (D == 128 ? 2 * i + (w >> 1) : w));
      blk8[s][i] = (int64_t)(id * (uint32_t)blk_bytes);
      const uint64_t p = reinterpret_cast<uint64_t>(a.scales) + 2 * (id * (uint32_t)a.hkv + g);
      sc8[s][i] = *reinterpret_cast<const __attribute__((address_space(4))) uint32_t*>(p & ~uint64_t(3)) >>
                  (8 * (uint32_t(p) & 2));
    }
  };
  // The wave-uniform address in scalar registers, the lane's offset in a vector one.
  // Steps past the last are loads of nothing: no branch splits the code around them.
  auto raw16 = [](const char* base, uint32_t off, bool load) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(base), (short)0, load ? kHeadBytes : 0, 0x00020000);
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, STREAM ? kCachePolicyNonTemporal : 0));
  };
  auto load_k8 = [&](int s, bool load) {
#pragma unroll
    for (int i = 0; i < NR; ++i) rk[i] = raw16(kbase + blk8[s][i], koff8, load);
  };
  auto load_v8 = [&](int s, bool load) {
#pragma unroll
    for (int i = 0; i < NR; ++i) rv[i] = raw16(vbase + blk8[s][i], piece_off + 16 * lane, load);
  };
  auto store_k8 = [&](int s) {
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const float sc = scale8(sc8[s][i] & 255);
      // units of 16 bytes; a piece fills two 32-dim groups (128 units) of the tile
      __bf16* p = &sm.k[s][8 * (128 * (4 * i + w))];
      st16(p + 8 * kdst8, bf16_of_e4m3(rk[i][0], rk[i][1], sc));
      st16(p + 8 * (kdst8 ^ 1), bf16_of_e4m3(rk[i][2], rk[i][3], sc));
    }
  };
  uint32_t scv[NR];  // scales of the V^T to store
  auto store_v8 = [&](int s) {
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const float sc = scale8(scv[i] >> 8 & 255);
      const int sw = vswz(lane);  // vswz(64 + d) == vswz(d)
      __bf16* p = &sm.v[s][8 * (128 * (4 * i + w) + 2 * lane)];
      st16(p + 8 * sw, bf16_of_e4m3(rv[i][0], rv[i][1], sc));
      st16(p + 8 * (1 - sw), bf16_of_e4m3(rv[i][2], rv[i][3], sc));
    }
  };

  // KV4 staging.  Of K a lane takes part4 (a quarter of the dims) of token tok4; the low
  // lane bits choose the slot so that eight neighbouring lanes write in distinct banks.
  // Of V^T, unit4: at head_dim 128 16 bytes, dims 32 c + i and 32 c + 16 + i; at 64 one dim.
  constexpr int kScaleRows = D / kKeyGroup + 1;
  constexpr int NW = D / 32;  // words of a lane's K, and of its V^T
  typedef uint32_t raw4 __attribute__((ext_vector_type(NW)));
  raw4 rk4, rv4;
  uint32_t sk4 = 0, sv4 = 0;  // scale bytes of the raw K and V^T
  int64_t id4[2];             // the block of this wavefront, times hkv, + g: by step % 2
  const int pos4 = (lane & 1) | (lane & 6) << 1 | (lane >> 2 & 2), tok4 = key_slot_pos(pos4);
  const int part4 = D == 128 ? lane >> 4 : (lane >> 5) << 1 | (lane >> 4 & 1);
  const int row4 = D == 128 ? part4 : part4 >> 1;  // 32-dim group
  const uint32_t koff4 = tok4 * (D / 2) + part4 * (D / 8);
  const uint32_t kdst4 = 64 * row4 + 4 * pos4, kswz4 = (pos4 >> 2) & 3;
  const int dim4 = D == 128 ? (lane >> 4) * 32 + (lane & 15) : (lane >> 5) * 32 + (lane & 31);
  const uint32_t voff4 = D == 128 ? 16 * lane : (lane >> 5) * 256 + (lane & 15) * 16 + (lane >> 4 & 1) * 8;
  auto step_blocks4 = [&](int t0, int s) {
    const int jb = t0 / kBlock;
    win.seek(jb);
    id4[s] = (int64_t)((uint64_t)(uint32_t)win.at(jb + w) * (uint32_t)a.hkv) + g;
  };
  auto raw_words = [](const uint8_t* base, uint32_t off, bool load) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(base), (short)0, load ? kHeadBytes : 0, 0x00020000);
    constexpr int policy = STREAM ? kCachePolicyNonTemporal : 0;
    if constexpr (D == 128) return __builtin_bit_cast(raw4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, policy));
    else return __builtin_bit_cast(raw4, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, policy));
  };
  auto raw_scale = [](const uint8_t* base, uint32_t off, bool load) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(base), (short)0, load ? kScaleRows * kBlock : 0, 0x00020000);
    return (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(r, off, 0, 0);
  };
  auto load_k4 = [&](int s, bool load) {
    rk4 = raw_words(reinterpret_cast<const uint8_t*>(a.kc) + id4[s] * kHeadBytes, koff4, load);
    sk4 = raw_scale(a.scales + id4[s] * (kScaleRows * kBlock), row4 * kBlock + tok4, load);
  };
  auto load_v4 = [&](int s, bool load) {
    rv4 = raw_words(reinterpret_cast<const uint8_t*>(a.vc) + id4[s] * kHeadBytes, voff4, load);
    sv4 = raw_scale(a.scales + id4[s] * (kScaleRows * kBlock), (kScaleRows - 1) * kBlock + (lane & 15), load);
  };
  auto store_k4 = [&](int s) {
    __bf16* p = &sm.k[s][8 * (w * (2 * D))];  // units of 16 bytes: 2 D a block
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const uint32_t unit = D == 128 ? i : 2 * (part4 & 1) + i;
      st16(p + 8 * (kdst4 + (unit ^ kswz4)), bf16_of_e2m1(rk4[i], exponent_byte(sk4, 0)));
    }
  };
  auto store_v4 = [&](int s) {
#pragma unroll
    for (int i = 0; i < NW / 2; ++i) {
      const int d = dim4 + 16 * i, sw = vswz(d);
      __bf16* p = &sm.v[s][8 * (w * (2 * D) + 2 * d)];
      st16(p + 8 * sw, bf16_of_e2m1(rv4[2 * i], 1.f));
      st16(p + 8 * (1 - sw), bf16_of_e2m1(rv4[2 * i + 1], 1.f));
    }
    if (lane < kBlock) sm.sv[s][kBlock * w + lane] = scale8(sv4);
  };

  // LDS operand addresses: per lane, the byte offset of its K unit for each
  // k-step (row j of a 32-key tile; the swizzle depends on the k-step) and
  // of its V^T unit; buffers, 32-key tiles and 32-dim tiles add constants, so
  // with the buffer known at compile time every operand read is one
  // register plus an immediate offset.
  uint32_t kofs[D / 16];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    const int pos = j % kBlock;
    kofs[ks] = 16u * (((j / kBlock) * (D / kKeyGroup) + ks / 2) * 64 + 4 * pos +
                      ((2 * (ks % 2) + hh) ^ ((pos >> 2) & 3)));
  }
  const uint32_t vofs = 16u * (2 * j + (hh ^ vswz(j)));  // vswz(32 dt + j) == vswz(j)
  auto lds_at = [](const __bf16* base, uint32_t byte_off) {
    return reinterpret_cast<const __bf16*>(reinterpret_cast<const char*>(base) + byte_off);
  };

  // S^T[key][row] of a step for the wave's 32 rows: NSUB independent 32-key chains.
  auto scores = [&](auto buf_c, f32x16 (&s)[NSUB]) {
    constexpr int buf = decltype(buf_c)::value;
#pragma unroll
    for (int u = 0; u < NSUB; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
    // MFMA i: k-step i / NSUB of 32-key chain i % NSUB
    lds_mfma_pipeline<D / 16 * NSUB, PA_LDS_PREFETCH>(
        [&](int i) { return lds_at(&sm.k[buf][32 * (i % NSUB) * D], kofs[i / NSUB]); },
        [&](int i, u32x4 k) { s[i % NSUB] = mfma32(as_bf16x8(k), qf[i / NSUB], s[i % NSUB]); });
  };
  // element e of tile u is key t0 + 32 u + perm32(8 (e / 4) + 4 hh + e % 4); perm32
  // moves hh to bit 3, so the rest of the key is a constant
  auto mask = [&](int t0, f32x16 (&s)[NSUB]) {
    const int lim = apos - t0 - 8 * hh;
#pragma unroll
    for (int u = 0; u < NSUB; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        s[u][e] = 32 * u + perm32(8 * (e >> 2) + (e & 3)) <= lim ? s[u][e] : kNegInf;
  };
  auto rowmax = [&](const f32x16 (&s)[NSUB]) {
    float mx = fmaxf(s[0][0], s[0][1]);
#pragma unroll
    for (int u = 0; u < NSUB; ++u)
#pragma unroll
      for (int e = (u == 0 ? 2 : 0); e < 16; e += 2) mx = fmaxf(fmaxf(mx, s[u][e]), s[u][e + 1]);
    return max_halves(mx);
  };
  // Move the reference to the running max: the output and row sums so far are
  // rescaled.
  auto rebase = [&](float mx) {
    const float mnew = fmaxf(m, mx);
    const float mcn = mnew == kNegInf ? 0.f : mnew * c;
    const float alpha = m == kNegInf ? 0.f : fast_exp2(mc - mcn);
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[dt][e] *= alpha;
    m = mnew;
    mc = mcn;
  };
  // Probabilities of a step as bf16 B operands: p[u][kk] holds keys
  // 32 u + 16 kk + 8 hh + 0..7 (the perm32 order makes them consecutive).
  // Returns this lane's row sum: the bf16 probabilities the PV product uses,
  // two per v_dot2, in two chains.  KV8 sums the float32 probabilities, so that the
  // log-sum-exp of rows of few keys does not carry the rounding to bf16.  The product
  // keeps it in both: the matrix instruction takes bf16, and a second term for what the
  // first leaves would double the PV product for outputs that are rounded to bf16 anyway
  // (off the exact ones by 1.7e-3 with that rounding alone, 1.8e-3 to 2.0e-3 with both).
  // KV4: as KV8; the products take the probabilities times their tokens' value scales.
  auto exps = [&](const f32x16 (&s)[NSUB], bf16x8 (&p)[NSUB][2], int buf) {
    if constexpr (KV4) {
      // Scales of elements 4 e4 .. + 3 of tile u, keys 32 u + 16 (e4 / 2) + 8 hh +
      // 4 (e4 % 2) .. + 3: read one group ahead, no further (all at once they push other
      // values out of the registers).
      auto scales_of = [&](int i) {
        const int u = i / 4, e4 = i % 4;
        return *reinterpret_cast<const f32x4*>(&sm.sv[buf][32 * u + 16 * (e4 >> 1) + 4 * (e4 & 1) + 8 * hh]);
      };
      float l0 = 0.f, l1 = 0.f;
      f32x4 next = scales_of(0);
#pragma unroll
      for (int i = 0; i < 4 * NSUB; ++i) {
        const f32x4 sv = next;
        if (i + 1 < 4 * NSUB) next = scales_of(i + 1);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int u = i / 4, e = 4 * (i % 4) + k;
          const float x = fast_exp2(fmaf(s[u][e], c, -mc));
          p[u][e >> 3][e & 7] = (__bf16)times_scale(x, sv[k]);
          (e < 8 ? l0 : l1) += x;
        }
        // formed here: behind the look at the sum, exponentials and scales would all wait
        // in registers
        if (i % 2) {
          u32x4 t = __builtin_bit_cast(u32x4, p[i / 4][i % 4 / 2]);
          asm volatile("" : "+v"(t), "+v"(l0), "+v"(l1));
          p[i / 4][i % 4 / 2] = as_bf16x8(t);
        }
      }
      return l0 + l1;
    } else if constexpr (KV8) {
      float l0 = 0.f, l1 = 0.f;
#pragma unroll
      for (int u = 0; u < NSUB; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = fast_exp2(fmaf(s[u][e], c, -mc));
          p[u][e >> 3][e & 7] = (__bf16)x;
          (e < 8 ? l0 : l1) += x;
        }
      return l0 + l1;
    } else {
#pragma unroll
      for (int u = 0; u < NSUB; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) p[u][e >> 3][e & 7] = (__bf16)fast_exp2(fmaf(s[u][e], c, -mc));
      float l0 = 0.f, l1 = 0.f;
#pragma unroll
      for (int u = 0; u < NSUB; ++u) {
        l0 = add_bf16x8(p[u][0], l0);
        l1 = add_bf16x8(p[u][1], l1);
      }
      return l0 + l1;
    }
  };
  // The reference only has to keep the probabilities in range (their relative
  // precision does not depend on it), and the row sum, which is needed
  // anyway, shows when it does not: no step looks for its maximum until a sum
  // exceeds kMaxSum (or is NaN, or a row has no reference yet); then the
  // wavefront moves the reference and forms the step's probabilities again.
  // Without the maximum of every step (20 of ~120 VALU instructions) prefill of
  // 64 requests on a 2048-token prefix takes 1.49 ms per append and call against
  // 1.53, 28/4-head prompts of 4000-12000 tokens 0.777 against 0.794, 24 requests at
  // head_dim 64, whose registers then allow a third wavefront per SIMD, 105 us
  // against 115.
  // Sums of 2^8 leave the float32 sums the room they have where each step looks for
  // its maximum and moves the reference beyond 2^8 (a value near the type's largest,
  // times its probability, stays finite).
  constexpr float kMaxSum = 256.f;
  auto probs = [&](const f32x16 (&s)[NSUB], bf16x8 (&p)[NSUB][2], int buf) {
    float sum = exps(s, p, buf);
    if (__any(!(sum <= kMaxSum) || m == kNegInf)) {
      rebase(rowmax(s));
      sum = exps(s, p, buf);
    }
    l += sum;
  };
  auto pv = [&](auto buf_c, const bf16x8 (&p)[NSUB][2]) {
    constexpr int buf = decltype(buf_c)::value;
    // MFMA i: dims 32 (i % DT) .. of keys 16 (i / DT) .. (16-key half i / DT)
    constexpr int DT = D / 32;
    lds_mfma_pipeline<2 * NSUB * DT, PA_LDS_PREFETCH>(
        [&](int i) { return lds_at(&sm.v[buf][(i / DT) * BLK + 512 * (i % DT)], vofs); },
        [&](int i, u32x4 v) {
          acc[i % DT] = mfma32(as_bf16x8(v), p[(i / DT) / 2][(i / DT) % 2], acc[i % DT]);
        });
  };
  // Values of keys at or past kend in the last step: zero (never-written cache
  // slots may hold anything, and 0 * NaN would reach the output).
  auto zero_tail = [&](int t0, int buf) {
    const int nz = t0 + KT - kend;
    for (int x = tid; x < D * nz; x += 256) {
      const int d = x % D, k = kend - t0 + x / D;
      const int b = k / kBlock, kk = k % kBlock;
      sm.v[buf][b * BLK + 8 * (2 * d + ((kk >> 3) ^ vswz(d))) + (kk & 7)] = (__bf16)0.f;
    }
  };

  const int ntiles = kend > kv0 ? (kend - kv0 + KT - 1) / KT : 0;
  // steps [0, n_plain) need no causal or tail mask for any row of the item
  const int n_plain = min(ntiles, max(0, (wg_amin + 1 - kv0) / KT));
  if (ntiles > 0) {
    // blk[t % 2]: byte offsets of step t's blocks, found two steps ahead
    // (for the K copy) and used again one step ahead (for the V^T copy)
    int64_t blk[2][NB] = {};
    if constexpr (KV8) {
      step_blocks8(kv0, 0);
      load_k8(0, true);
      load_v8(0, true);
#pragma unroll
      for (int i = 0; i < NR; ++i) scv[i] = sc8[0][i];
      store_k8(0);
      store_v8(0);
      if (ntiles > 1) {
        step_blocks8(kv0 + KT, 1);
        load_k8(1, true);
        load_v8(1, true);  // stored in step 0
        store_k8(1);
        step_blocks8(kv0 + KT * min(2, ntiles - 1), 0);
        load_k8(0, ntiles > 2);
      }
    } else if constexpr (KV4) {
      step_blocks4(kv0, 0);
      load_k4(0, true);
      load_v4(0, true);
      store_k4(0);
      store_v4(0);
      if (ntiles > 1) {
        step_blocks4(kv0 + KT, 1);
        load_k4(1, true);
        load_v4(1, true);  // stored in step 0
        store_k4(1);
        step_blocks4(kv0 + KT * min(2, ntiles - 1), 0);
        load_k4(0, ntiles > 2);
      }
    } else {
      step_blocks(kv0, blk[0]);
      issue_k(blk[0], 0);
      issue_v(blk[0], 0);
      if (ntiles > 1) {
        step_blocks(kv0 + KT, blk[1]);
        issue_k(blk[1], 1);
      }
      wait_vmem();
    }
    __syncthreads();
    // Wavefronts without rows (items of fewer than kTileRows rows) only help
    // with the copies and pass the barriers.
    const bool active = FULL || w * 32 < nrows;
    f32x16 s[NSUB];
    using B0 = std::integral_constant<int, 0>;
    using B1 = std::integral_constant<int, 1>;
    if (active) {
      scores(B0{}, s);
      if (n_plain == 0) mask(kv0, s);
      rebase(rowmax(s));
    }
    __syncthreads();  // K buffer 0 is refilled next

    // KV8 and KV4: blocks8 finds step t + 3's blocks, stage8 puts K of step t + 2 and V^T of step
    // t + 1 into LDS (past the last step: unused buffers) and the next on their way
    auto blocks8 = [&](int t, auto buf_c) {
      constexpr int buf = decltype(buf_c)::value;
      if constexpr (KV4) {
        // step t + 3's where step t + 1's were, whose V^T is on its way
        step_blocks4(kv0 + KT * min(t + 3, ntiles - 1), 1 - buf);
        return;
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) scv[i] = sc8[1 - buf][i];  // of step t + 1
      step_blocks8(kv0 + KT * min(t + 3, ntiles - 1), 1 - buf);
    };
    auto stage8 = [&](int t, auto buf_c) {
      constexpr int buf = decltype(buf_c)::value;
      if constexpr (KV4) {
        store_v4(1 - buf);
        store_k4(buf);
        load_v4(buf, t + 2 < ntiles);
        load_k4(1 - buf, t + 3 < ntiles);
        return;
      }
      store_v8(1 - buf);
      store_k8(buf);
      load_v8(buf, t + 2 < ntiles);  // whose blocks were found one step earlier
      load_k8(1 - buf, t + 3 < ntiles);
    };
    // One pipelined step: softmax + PV of step t, scores of step t + 1.
    // buf_c = t % 2, the LDS buffer pair of step t (a compile-time constant).
    auto step = [&](int t, auto mask_next, auto buf_c) {
      constexpr int buf = decltype(buf_c)::value;
      const int t0 = kv0 + KT * t;
      if constexpr (!STAGED) {
        if (t + 2 < ntiles) {
          step_blocks(t0 + 2 * KT, blk[buf]);
          issue_k(blk[buf], buf);
        }
        issue_v(blk[1 - buf], 1 - buf);  // blocks of step t + 1, found one step earlier
      }
      if constexpr (STAGED) blocks8(t, buf_c);
      bf16x8 p[NSUB][2];
      f32x16 sn[NSUB];
      probs(s, p, buf);
      // The matrix section runs at raised issue priority: of the two
      // wavefronts sharing a SIMD, the one issuing MFMAs goes first and the
      // other's softmax VALU work fills the remaining issue slots.
      __builtin_amdgcn_s_setprio(1);
      scores(std::integral_constant<int, 1 - buf>{}, sn);
      // keep the row-sum additions in this region, where they overlap the
      // score MFMAs, instead of letting them sink past the barrier
      asm volatile("" : "+v"(l));
      // The conversions go beside the matrix instructions (12 prompts of 512 tokens at
      // head_dim 64 98.5 us, 101.9 at the step's start; head_dim 128 even).
      if constexpr (STAGED) stage8(t, buf_c);
      pv(buf_c, p);
      __builtin_amdgcn_s_setprio(0);
      if constexpr (decltype(mask_next)::value) mask(t0 + KT, sn);
      if constexpr (!STAGED) wait_vmem();  // KV8: the barrier waits for the stores into LDS
      __syncthreads();
#pragma unroll
      for (int u = 0; u < NSUB; ++u) s[u] = sn[u];
    };
    auto idle_step = [&](int t, auto buf_c) {
      if constexpr (STAGED) {
        blocks8(t, buf_c);
        stage8(t, buf_c);
      } else {
        constexpr int buf = decltype(buf_c)::value;
        const int t0 = kv0 + KT * t;
        if (t + 2 < ntiles) {
          step_blocks(t0 + 2 * KT, blk[buf]);
          issue_k(blk[buf], buf);
        }
        issue_v(blk[1 - buf], 1 - buf);
        wait_vmem();
      }
      __syncthreads();
    };
    // steps [t, lim) with the given masking, two at a time so that each
    // step's buffer pair is a compile-time constant
    auto run = [&](int& t, int lim, auto mask_next) {
      if (t < lim && (t & 1)) step(t++, mask_next, B1{});
      for (; t + 1 < lim; t += 2) {
        step(t, mask_next, B0{});
        step(t + 1, mask_next, B1{});
      }
      if (t < lim) step(t++, mask_next, B0{});
    };
    int t = 0;
    if (active) {
      // step t masks the scores of step t + 1: unmasked while t + 1 < n_plain
      run(t, min(n_plain, ntiles) - 1, std::false_type{});
      run(t, ntiles - 1, std::true_type{});
    } else {
      for (; t + 2 < ntiles; t += 2) {
        idle_step(t, B0{});
        idle_step(t + 1, B1{});
      }
      if (t + 1 < ntiles) idle_step(t++, B0{});
    }
    // last step: softmax + PV only
    const int t0 = kv0 + KT * t;
    bf16x8 p[NSUB][2];
    if (active) probs(s, p, t & 1);
    if (!KV4 && t0 + KT > kend) {  // KV4: codes are numbers, and those keys' products zero
      zero_tail(t0, t & 1);
      __syncthreads();
    }
    if (active) {
      if (t & 1) pv(B1{}, p);
      else pv(B0{}, p);
    }
  }

  l += wave_xor(l, 32);
  if (!valid) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const float lse_v = l > 0.f ? kLn2 * (mc + __log2f(l)) : kNegInf;
  if (part < 0) {
    __bf16* op = a.out + ((int64_t)(qs + qi) * a.hq + hq) * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int d = 32 * dt + 8 * q4 + 4 * hh;
        __bf16 o4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(acc[dt][4 * q4 + e] * inv);
        *reinterpret_cast<u32x2*>(op + d) = __builtin_bit_cast(u32x2, o4);
      }
    if (a.lse && hh == 0) a.lse[(int64_t)(qs + qi) * a.hq + hq] = lse_v;
  } else {
    float* op = a.ws_o + (int64_t)part * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int d = 32 * dt + 8 * q4 + 4 * hh;
        f32x4 o4;
#pragma unroll
        for (int e = 0; e < 4; ++e) o4[e] = acc[dt][4 * q4 + e] * inv;
        *reinterpret_cast<f32x4*>(op + d) = o4;
      }
    if (hh == 0) a.ws_lse[part] = l == l ? lse_v : l;
  }
}

// Row item: one wavefront, up to 16 * NC rows (NC 16-column MFMA tiles that
// share every K and V^T operand), keys [kv0, kv1).  Decode items hold a
// sequence's G rows (NC = 1); verification items hold up to 32 of its
// n_q * G rows (NC = 2), so the keys are streamed from memory once per 32
// rows.  Sequences with more rows use tile items.
template <int D, int NC>
__device__ __forceinline__ void row_item(const int32_t* it, int g, int poff, const AttnArgs& a) {
  constexpr int KS = D / 32;  // k-steps of the QK product (32 dims each)
  constexpr int DT = D / 16;  // 16-row tiles of O^T
  const int r = it[I_SEQ];
  if (r < 0) return;
  const int row0 = it[I_ROW0], nrows = it[I_NROWS];
  const int kv0 = it[I_KV0], part = it[I_PART] < 0 ? -1 : it[I_PART] + poff;
  const int lane = threadIdx.x & 63, j = lane & 15, g4 = lane >> 4;
  const int L = a.seq_lens[r];
  const int qs = a.cu_q[r], n = a.cu_q[r + 1] - qs;
  // at most kRowItemBlocks blocks per item (the planner's limit; the clamp
  // keeps every table read inside the item's span)
  const int kv1 = min(min(it[I_KV1], L), kv0 + kRowItemBlocks * kBlock);
  const int G = a.group;

  // column j of tile c is the item's row 16 c + j
  bool valid[NC];
  int qi[NC], hq[NC], apos[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    valid[c] = 16 * c + j < nrows;
    const int rho = row0 + 16 * c + j;
    qi[c] = rho / G;
    hq[c] = g * G + (rho - qi[c] * G);
    apos[c] = valid[c] ? L - n + qi[c] : -1;
  }
  const int amin = L - n + row0 / G;  // smallest position among the item's rows

  bf16x8 qf[NC][KS];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const __bf16* qp = a.q + ((int64_t)(qs + qi[c]) * a.hq + hq[c]) * D + 8 * g4;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[c][ks] = as_bf16x8(valid[c] ? ld16(qp + 32 * ks) : zero16());
  }
  f32x4 acc[NC][DT];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[c][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float cs = a.scale_log2;
  float m[NC], mc[NC], l[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) m[c] = kNegInf, mc[c] = 0.f, l[c] = 0.f;

  const int32_t* bt = a.bt + (int64_t)r * a.max_blocks;
  const int64_t blk_k = (int64_t)a.hkv * kBlock * D, head_k = (int64_t)g * kBlock * D;
  const int64_t blk_v = (int64_t)a.hkv * D * kBlock, head_v = (int64_t)g * D * kBlock;
  // K operand row j of score tile tt holds key 8 * (j / 4) + 4 * tt + j % 4,
  // so each lane's score elements are eight consecutive keys (8 g4 .. + 7).

  // One register set for K and one for V^T: the next step's K loads are
  // issued as soon as the score MFMAs have consumed K, and its V^T loads as
  // soon as the PV MFMAs have consumed V^T, so HBM reads overlap the softmax
  // and the MFMAs of the current step.  The loads are non-temporal (private
  // keys are read once).  All loads are in bounds (a missing second block
  // aliases the first).
  u32x4 kreg[2][KS], vreg[DT];
  int b0 = 0, b1 = 0;
  BlockSpan win;
  win.init(bt, a.max_blocks, kv0 / kBlock);
  auto blocks_of = [&](int t0) {
    const int jb = t0 / kBlock;
    b0 = clamp_block(win.get(jb), a.num_blocks);
    b1 = t0 + 16 < kv1 ? clamp_block(win.get(jb + 1), a.num_blocks) : b0;
  };
  // That key sits in block j / 8 at slot position 8 tt + j % 8 (the grouped
  // key layout): each load reads, per block, eight
  // consecutive 64-byte slot rows of one 32-dim group, 512 contiguous bytes.
  auto load_k = [&]() {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int blk = j < 8 ? b0 : b1;
      const __bf16* p = a.kc + blk * blk_k + head_k + (8 * tt + (j & 7)) * kKeyGroup + 8 * g4;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        kreg[tt][ks] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + kBlock * kKeyGroup * ks));
    }
  };
  auto load_v = [&]() {
    const __bf16* p = a.vc + (g4 < 2 ? b0 : b1) * blk_v + head_v + j * kBlock + 8 * (g4 & 1);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) vreg[dt] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 16 * kBlock * dt));
  };

  if (kv0 < kv1) {
    blocks_of(kv0);
    load_k();
    load_v();
  }
  for (int t0 = kv0; t0 < kv1; t0 += 32) {
    const bool more = t0 + 32 < kv1;
    f32x4 s[NC][2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        f32x4 acc_s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc_s = mfma16(as_bf16x8(kreg[tt][ks]), qf[c][ks], acc_s);
        s[c][tt] = acc_s;
      }
    if (more) {
      blocks_of(t0 + 32);
      load_k();
    }
    // Lane (j, g4), element e of score tile tt holds key t0 + 8 g4 + 4 tt + e.
    const bool masked = t0 + 31 > amin || !more;  // wave-uniform
    if (masked) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = t0 + 8 * g4 + 4 * tt + e;
            s[c][tt][e] = (key <= apos[c] && key < kv1) ? s[c][tt][e] : kNegInf;
          }
      // zero values of keys at or past kv1 (slots that may never have been written)
      const int keep = min(max(kv1 - (t0 + 8 * g4), 0), 8);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vreg[dt] = keep_bf16(vreg[dt], keep);
    }
    bf16x8 pb[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float mx = fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3]));
      mx = fmaxf(mx, fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3])));
      mx = fmaxf(mx, wave_xor(mx, 16));
      mx = fmaxf(mx, wave_xor(mx, 32));
      if (__any(mx != kNegInf && (m[c] == kNegInf || mx * cs > mc[c] + 8.f))) {
        const float mnew = fmaxf(m[c], mx);
        const float mcn = mnew == kNegInf ? 0.f : mnew * cs;
        const float alpha = m[c] == kNegInf ? 0.f : fast_exp2(mc[c] - mcn);
        l[c] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[c][dt] *= alpha;
        m[c] = mnew;
        mc[c] = mcn;
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = fast_exp2(fmaf(s[c][tt][e], cs, -mc[c]));
          l[c] += p;
          pb[c][4 * tt + e] = (__bf16)p;
        }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c][dt] = mfma16(as_bf16x8(vreg[dt]), pb[c], acc[c][dt]);
    if (more) load_v();
  }

#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += wave_xor(l[c], 16);
    l[c] += wave_xor(l[c], 32);
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (!valid[c]) continue;
    const float inv = l[c] > 0.f ? 1.f / l[c] : 0.f;
    const float lse_v = l[c] > 0.f ? kLn2 * (mc[c] + __log2f(l[c])) : kNegInf;
    if (part < 0) {
      __bf16* op = a.out + ((int64_t)(qs + qi[c]) * a.hq + hq[c]) * D + 4 * g4;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        __bf16 o4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(acc[c][dt][e] * inv);
        *reinterpret_cast<u32x2*>(op + 16 * dt) = __builtin_bit_cast(u32x2, o4);
      }
      if (a.lse && g4 == 0) a.lse[(int64_t)(qs + qi[c]) * a.hq + hq[c]] = lse_v;
    } else {
      const int prow = part + 16 * c + j;
      float* op = a.ws_o + (int64_t)prow * D + 4 * g4;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(op + 16 * dt) = acc[c][dt] * inv;
      if (g4 == 0) a.ws_lse[prow] = l[c] == l[c] ? lse_v : l[c];
    }
  }
}

// A row item's result for the row in this lane's column: output and log-sum-exp of
// (token, q-head) where prow < 0, else partial row prow.
template <int D>
__device__ __forceinline__ void store_row(const AttnArgs& a, const f32x4 (&acc)[D / 16], float l, float mc,
                                          int token, int hq, int prow, int g4) {
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const float lse_v = l > 0.f ? kLn2 * (mc + __log2f(l)) : kNegInf;
  if (prow < 0) {
    __bf16* op = a.out + ((int64_t)token * a.hq + hq) * D + 4 * g4;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      __bf16 o4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(acc[dt][e] * inv);
      *reinterpret_cast<u32x2*>(op + 16 * dt) = __builtin_bit_cast(u32x2, o4);
    }
    if (a.lse && g4 == 0) a.lse[(int64_t)token * a.hq + hq] = lse_v;
  } else {
    float* op = a.ws_o + (int64_t)prow * D + 4 * g4;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(op + 16 * dt) = acc[dt] * inv;
    if (g4 == 0) a.ws_lse[prow] = l == l ? lse_v : l;
  }
}

// Row item over the 8-bit cache: as row_item, in steps of 64 keys (four blocks),
// so that every load is 16 bytes per lane of 64 contiguous bytes of a key or a
// dimension's 16 keys.  Score tile tt takes tokens 4 tt .. 4 tt + 3 of each of the
// four blocks: row j is token 4 tt + j % 4 of block j / 4, and lane (j, g4)'s
// elements are keys 4 tt + e of block g4, the block whose values the lane holds as
// A operand of the PV product (16 keys of dimension 16 dt + j: two k-steps).  The
// score's k-steps take dims 64 c + 16 g4 + 8 u .. + 7, the halves u of a lane's load.
// The 4-bit cache: a lane takes 16 bytes of a key (head_dim 64: 8) that share a scale, and
// 16 keys of dims 32 i + j and 32 i + 16 + j.  Score tiles hold the same tokens: four
// neighbouring ones' keys are 256 contiguous bytes of a load (of tokens 4 apart, 64 bytes
// at a time, 64 sequences of 2000-8000 keys at head_dim 64 took 56 us instead of 44, 32 of
// 4000-8000 28/4 heads 31 and 27.5).
// With kItemJoin the workgroup's four wavefronts hold the same rows over adjacent
// keys: they leave their accumulators, references and sums in LDS, and each combines a
// quarter of the output dims and writes them.
template <int D, int NC>
struct JoinSmem {
  f32x4 acc[4][NC][D / 16][64];  // [wavefront][column tile][16 dims][lane]
};
struct JoinStat {
  float mc, l;  // reference (scaled; minus infinity without a key) and sum of a row
};

template <int D, int NC, int BITS, bool AHEAD, bool TWICE>
__device__ __forceinline__ void row_item8(const int32_t* it, int g, int poff, const AttnArgs& a,
                                          JoinSmem<D, NC>& sm, JoinStat (&stat)[4][2][16]) {
  constexpr bool KV4 = BITS == 4;
  constexpr int KC = D / 64;  // 64-dim groups of a key
  constexpr int DT = D / 16;  // 16-row tiles of O^T
  constexpr int kStep = kKeyStep8;
  constexpr int kScaleRows = D / kKeyGroup + 1;
  const int r = it[I_SEQ];
  if (r < 0) return;
  const int row0 = it[I_ROW0], nrows = it[I_NROWS];
  const int kv0 = it[I_KV0], part = it[I_PART] < 0 ? -1 : it[I_PART] + poff;
  const int lane = threadIdx.x & 63, j = lane & 15, g4 = lane >> 4;
  const int L = a.seq_lens[r];
  const int qs = a.cu_q[r], n = a.cu_q[r + 1] - qs;
  // at most kRowItemBlocks blocks per item, as in row_item
  const int kv1 = min(min(it[I_KV1], L), kv0 + kRowItemBlocks * kBlock);
  const int G = a.group;

  bool valid[NC];
  int qi[NC], hq[NC], apos[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    valid[c] = 16 * c + j < nrows;
    const int rho = row0 + 16 * c + j;
    qi[c] = rho / G;
    hq[c] = g * G + (rho - qi[c] * G);
    apos[c] = valid[c] ? L - n + qi[c] : -1;
  }
  const int amin = L - n + row0 / G;

  bf16x8 qf[NC][2 * KC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const __bf16* qp = a.q + ((int64_t)(qs + qi[c]) * a.hq + hq[c]) * D + (KV4 ? D / 4 : 16) * g4;
#pragma unroll
    for (int ks = 0; ks < 2 * KC; ++ks)
      qf[c][ks] = as_bf16x8(valid[c] ? ld16(qp + (KV4 ? 8 * ks : 64 * (ks / 2) + 8 * (ks % 2))) : zero16());
  }
  f32x4 acc[NC][DT];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[c][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float cs = a.scale_log2;
  float m[NC], mc[NC], l[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) m[c] = kNegInf, mc[c] = 0.f, l[c] = 0.f;

  // AHEAD: two register sets of K and V^T; a step loads the next one's before it uses its
  // own, so a whole step hides the memory's latency (24 sequences of 8192-20480 keys 121
  // us, 5.9 TB/s, against 145 with one set and three wavefronts per SIMD instead of two).
  // Over the 4-bit cache those 24 sequences take 70 us, 5.4 TB/s; at head_dim 64 one set and
  // three wavefronts are enough there (64 sequences of 2000-8000 keys 39 us, 44 with two).
  // Beside tiles or two-tile items, which leave two wavefronts anyway, one set, reloaded as
  // in row_item, is as good or better: 128 decode requests on 4096 shared keys 48.6 us, 51.1
  // with two, 32 verifications on 16384 158 and 170 (an item ahead of the other that reads
  // its keys finds them in no cache).  Blocks at or past kv1 read the item's last block again.
  constexpr int NB = AHEAD ? 2 : 1;
  const uint8_t* kc = reinterpret_cast<const uint8_t*>(a.kc);
  const uint8_t* vc = reinterpret_cast<const uint8_t*>(a.vc);
  const int last = kv1 > kv0 ? (kv1 - 1) / kBlock : kv0 / kBlock;
  BlockSpan win;
  win.init(a.bt + (int64_t)r * a.max_blocks, a.max_blocks, kv0 / kBlock);
  auto block_of = [&](int jb) {  // per lane
    const int id = __shfl(win.ids, (min(jb, last) - win.base) & 63, 64);
    return (int64_t)clamp_block(id, a.num_blocks) * a.hkv + g;
  };
  // TWICE: another item reads the same keys (the other rows of a sequence of more than
  // kRowItemRows), so the loads leave them in the caches: 32 sequences of 3000 keys, 5
  // tokens, 64/8 heads 64 us against 70 with non-temporal ones; 256 decode requests, whose
  // keys are read once, 74 against 86 without those.
  auto raw16 = [](const uint8_t* p) {
    if constexpr (TWICE) return ld16(p);
    else return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  };
  // registers of a load: KV8 kreg[tt][c] and vreg[dt], KV4 kreg[tt][0] (head_dim 64: two
  // of its words) and vreg[i]
  constexpr int KR = KV4 ? 1 : KC, VR = KV4 ? DT / 2 : DT;
  u32x4 kreg[NB][4][KR], vreg[NB][VR];
  uint32_t ek[NB] = {}, ev[NB] = {};
  u32x4 ek4[NB], ev4[NB];  // KV4: scales of a block's 16 keys (of the lane's dims) and values
  auto load_k = [&](int t0, int s) {
    const int64_t b = block_of(t0 / kBlock + (j >> 2));
    if constexpr (KV4) {
      const uint8_t* p = kc + b * (kBlock * D / 2) + (j & 3) * (D / 2) + g4 * (D / 8);
#pragma unroll
      for (int tt = 0; tt < 4; ++tt) {
        if constexpr (D == 128) {
          kreg[s][tt][0] = raw16(p + 4 * tt * (D / 2));
        } else {
          u32x2 x;
          if constexpr (TWICE) x = *reinterpret_cast<const u32x2*>(p + 4 * tt * (D / 2));
          else x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p + 4 * tt * (D / 2)));
          kreg[s][tt][0][0] = x[0], kreg[s][tt][0][1] = x[1];
        }
      }
      ek4[s] = ld16(a.scales + b * (kScaleRows * kBlock) + (D == 128 ? g4 : g4 >> 1) * kBlock);
      return;
    }
    const uint8_t* p = kc + b * (kBlock * D) + (j & 3) * 64 + 16 * g4;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int c = 0; c < KR; ++c)
        kreg[s][tt][c] = raw16(p + 1024 * c + 256 * tt);
    ek[s] = a.scales[2 * b];
  };
  auto load_v = [&](int t0, int s) {
    const int64_t b = block_of(t0 / kBlock + g4);
    if constexpr (KV4) {
      const uint8_t* p = vc + b * (kBlock * D / 2) + j * kBlock;
#pragma unroll
      for (int i = 0; i < VR; ++i) vreg[s][i] = raw16(p + 256 * i);
      ev4[s] = ld16(a.scales + b * (kScaleRows * kBlock) + (kScaleRows - 1) * kBlock);
      return;
    }
    const uint8_t* p = vc + b * (kBlock * D) + j * kBlock;
#pragma unroll
    for (int dt = 0; dt < VR; ++dt)
      vreg[s][dt] = raw16(p + 256 * dt);
    ev[s] = a.scales[2 * b + 1];
  };

  if (kv0 < kv1) {
    load_k(kv0, 0);
    load_v(kv0, 0);
  }
  // the step at t0, its K and V^T in register set b
  auto step = [&](int t0, auto b) {
    constexpr int cur = decltype(b)::value, next = AHEAD ? 1 - cur : 0;
    const bool more = t0 + kStep < kv1;
    if (AHEAD && more) {
      load_k(t0 + kStep, next);
      load_v(t0 + kStep, next);
    }
    f32x4 s[NC][4];
    const float sk = scale8(ek[cur]);
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
      for (int c = 0; c < NC; ++c) s[c][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 2 * KC; ++ks) {
        bf16x8 k;
        if constexpr (KV4) {
          k = as_bf16x8(bf16_of_e2m1(kreg[cur][tt][0][ks], exponent_byte(ek4[cur][tt] >> (8 * (j & 3)), 0)));
        } else {
          const u32x4 x = kreg[cur][tt][ks / 2];
          k = as_bf16x8(bf16_of_e4m3(x[2 * (ks % 2)], x[2 * (ks % 2) + 1], sk));
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) s[c][tt] = mfma16(k, qf[c][ks], s[c][tt]);
      }
    }
    if (!AHEAD && more) load_k(t0 + kStep, next);
    // Lane (j, g4), element e of score tile tt holds key t0 + 16 g4 + 4 tt + e.
    const bool masked = t0 + kStep - 1 > amin || !more;  // wave-uniform
    if (masked) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = t0 + 16 * g4 + 4 * tt + e;
            s[c][tt][e] = (key <= apos[c] && key < kv1) ? s[c][tt][e] : kNegInf;
          }
      // zero values of keys at or past kv1 (slots that may never have been written); KV4:
      // codes are numbers, and a probability of zero stays zero times any scale
      const int keep = kv1 - (t0 + 16 * g4);
#pragma unroll
      for (int k = 0; k < (KV4 ? 0 : 4); ++k) {
        const int b = min(max(keep - 4 * k, 0), 4);
        const uint32_t mask = b == 4 ? ~0u : (1u << (8 * b)) - 1u;
#pragma unroll
        for (int dt = 0; dt < VR; ++dt) vreg[cur][dt][k] &= mask;
      }
    }
    bf16x8 pb[NC][2];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float mx = kNegInf;
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
        mx = fmaxf(mx, fmaxf(fmaxf(s[c][tt][0], s[c][tt][1]), fmaxf(s[c][tt][2], s[c][tt][3])));
      mx = fmaxf(mx, wave_xor(mx, 16));
      mx = fmaxf(mx, wave_xor(mx, 32));
      if (__any(mx != kNegInf && (m[c] == kNegInf || mx * cs > mc[c] + 8.f))) {
        const float mnew = fmaxf(m[c], mx);
        const float mcn = mnew == kNegInf ? 0.f : mnew * cs;
        const float alpha = m[c] == kNegInf ? 0.f : fast_exp2(mc[c] - mcn);
        l[c] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[c][dt] *= alpha;
        m[c] = mnew;
        mc[c] = mcn;
      }
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = fast_exp2(fmaf(s[c][tt][e], cs, -mc[c]));
          l[c] += p;
          if constexpr (KV4)
            pb[c][tt >> 1][4 * (tt & 1) + e] = (__bf16)times_scale(p, scale8(ev4[cur][tt] >> (8 * e) & 255));
          else
            pb[c][tt >> 1][4 * (tt & 1) + e] = (__bf16)p;  // as in a tile's exps
        }
    }
    const float sv = scale8(ev[cur]);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8 v;
        if constexpr (KV4) v = as_bf16x8(bf16_of_e2m1(vreg[cur][dt / 2][2 * (dt % 2) + u], 1.f));
        else v = as_bf16x8(bf16_of_e4m3(vreg[cur][dt][2 * u], vreg[cur][dt][2 * u + 1], sv));
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[c][dt] = mfma16(v, pb[c][u], acc[c][dt]);
      }
    if (!AHEAD && more) load_v(t0 + kStep, next);
  };
  using B0 = std::integral_constant<int, 0>;
  if constexpr (AHEAD) {
    using B1 = std::integral_constant<int, 1>;
    for (int t0 = kv0; t0 < kv1; t0 += 2 * kStep) {
      step(t0, B0{});
      if (t0 + kStep < kv1) step(t0 + kStep, B1{});
    }
  } else {
    for (int t0 = kv0; t0 < kv1; t0 += kStep) step(t0, B0{});
  }

#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += wave_xor(l[c], 16);
    l[c] += wave_xor(l[c], 32);
  }
  if (it[I_FLAGS] & kItemJoin) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int first[4];  // the wavefronts' first keys
#pragma unroll
    for (int v = 0; v < 4; ++v) first[v] = (it + (v - w) * kItemWords)[I_KV0];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (g4 == 0) stat[w][c][j] = {m[c] == kNegInf ? kNegInf : mc[c], l[c]};
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) sm.acc[w][c][dt][lane] = acc[c][dt];
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      JoinStat st[4];
      bool seen[4];
      float top = kNegInf;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        st[v] = stat[v][c][j];
        top = fmaxf(top, st[v].mc);
      }
      float sum = 0.f, f[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        // A wavefront whose keys the row does not see counts for nothing.  The others' sums
        // and outputs are multiplied by their weights where those are zero, too: one that is
        // not a number makes the row none, however low the wavefront's other scores lie.
        seen[v] = apos[c] >= first[v];
        f[v] = !seen[v] ? 0.f : st[v].mc == kNegInf ? 1.f : fast_exp2(st[v].mc - top);
        sum += seen[v] ? f[v] * st[v].l : 0.f;
      }
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
      const float lse_v = sum > 0.f ? kLn2 * (top + __log2f(sum)) : kNegInf;
      const int64_t row = (int64_t)(qs + qi[c]) * a.hq + hq[c];
      const int64_t prow = part + 16 * c + j;
#pragma unroll
      for (int i = 0; i < DT / 4; ++i) {
        const int dt = 4 * i + w;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const f32x4 x = sm.acc[v][c][dt][lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += seen[v] ? f[v] * x[e] : 0.f;
        }
        if (!valid[c]) continue;
        if (part < 0) {
          __bf16 o4[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) o4[e] = (__bf16)(o[e] * inv);
          *reinterpret_cast<u32x2*>(a.out + row * D + 16 * dt + 4 * g4) = __builtin_bit_cast(u32x2, o4);
        } else {
          *reinterpret_cast<f32x4*>(a.ws_o + prow * D + 16 * dt + 4 * g4) = o * inv;
        }
      }
      if (valid[c] && g4 == 0 && w == 0) {
        if (part >= 0) a.ws_lse[prow] = sum == sum ? lse_v : sum;
        else if (a.lse) a.lse[row] = lse_v;
      }
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (valid[c]) store_row<D>(a, acc[c], l[c], mc[c], qs + qi[c], hq[c], part < 0 ? -1 : part + 16 * c + j, g4);
}

// MIX bits: 1 = tile and shared items, 2 = row items of at most 16 rows,
// 4 = row items of up to 32 rows, 8 = wildcard workgroups (tail lists).
// Separate instantiations keep a pure prefill or pure decode launch from
// paying the other paths' registers and LDS, and a plan without tail lists
// from paying for the wildcard loop; a launch with only 16-row row items
// runs at three waves per SIMD, and so does every launch at head_dim 64, whose
// tiles fit 168 registers (24 requests' prefill 123 us against 138 with two).
// Over the 8-bit cache 16-row items at head_dim 128 take two sets of loads and two waves,
// and the kernels that hold more than one kind of item do not fit their registers: 20 to
// 56 spilled ones (MIX 6, 7, 15, at head_dim 64 9, too; the bf16 kernels none), stored and
// loaded outside the key loops, at head_dim 64 also once per item of the tail lists.  Over
// the 4-bit cache 2 to 6 spill at head_dim 128, all but MIX 2 at head_dim 64 4 to 71.
template <int D, int MIX, int BITS>
constexpr int waves_per_eu() {
  return (MIX == 2 && BITS == 16) || D == 64 ? 3 : kTileWavesPerEu;
}

template <int D, int MIX, int BITS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(waves_per_eu<D, MIX, BITS>()))) void attn_bf16_kernel(AttnArgs a) {
  const int32_t* plan = a.plan;
  // this workgroup's kv-head and template (the dispatch list follows the
  // header, so its word loads together with the header words); template
  // indices run over the shared, tile and row templates in that order
  const int wd = plan[kHeaderWords + blockIdx.x];
  const int g = wd >> kDispatchHeadShift, ti = wd & kDispatchIndexMask;
  const int n_shared = plan[H_N_SHARED_TMPL];
  const int n_tile = n_shared + plan[H_N_TILE_TMPL];  // templates before the row templates
  const int poff = g * plan[H_HEAD_PARTIAL];  // the kv-head's partial rows
  // 8 and 4 bits: tiles and joined row items use the same LDS
  constexpr bool kQuantised = BITS < 16;
  using Tile = TileSmem<D, kTileSub, BITS>;
  constexpr size_t kTileBytes = (MIX & 1) ? sizeof(Tile) : 0;
  constexpr size_t kJoinBytes = (MIX & 4) ? sizeof(JoinSmem<D, 2>) : (MIX & 2) ? sizeof(JoinSmem<D, 1>) : 0;
  __shared__ __align__(16) char lds8[kQuantised ? (kTileBytes > kJoinBytes ? kTileBytes : kJoinBytes) : 16];
  if constexpr (MIX & 1) {
    __shared__ Tile tile_lds;
    Tile* const tile_sm = kQuantised ? reinterpret_cast<Tile*>(lds8) : &tile_lds;
    Tile& sm = *tile_sm;
    if constexpr ((MIX & 8) != 0) {
      if (ti == kWildcard) {
        // Take tail items (full tiles) from this XCD queue's list, then from
        // the other queues' lists while any has items left.  Each list has its
        // own counter in the plan (device-scope atomics, one cache line each);
        // the last wildcard workgroup to finish resets them, so the plan serves
        // the next call on the stream as uploaded.
        __shared__ int claim_sh;
        uint32_t* ctr = reinterpret_cast<uint32_t*>(const_cast<int32_t*>(plan)) + plan[H_CTR_OFF];
        const int32_t* tab = plan + plan[H_TAIL_OFF];
        const int32_t* tiles = plan + plan[H_TILE_OFF] - n_shared * kItemWords;
        const int home = blockIdx.x % kXcdQueues;  // the XCD queue this workgroup runs in
        // next item of list q, or past its end (every thread calls this)
        auto claim = [&](int q) {
          if (threadIdx.x == 0)
            claim_sh = int(__hip_atomic_fetch_add(ctr + q * kCounterWords, 1u, __ATOMIC_RELAXED,
                                                  __HIP_MEMORY_SCOPE_AGENT));
          __syncthreads();  // also: every wavefront is done with the previous item's LDS
          const int c = __builtin_amdgcn_readfirstlane(claim_sh);
          __syncthreads();  // claim_sh is written again next round
          return c;
        };
        auto run = [&](int q, int c) {
          const int tw = plan[tab[q] + c];
          const int tg = tw >> kDispatchHeadShift;
          tile_item<D, kTileSub, BITS, false, true>(tiles + (tw & kDispatchIndexMask) * kItemWords, tg,
                                              tg * plan[H_HEAD_PARTIAL], a, sm);
        };
        for (;;) {
          const int c = claim(home);
          if (c >= tab[kXcdQueues + home]) break;
          run(home, c);
        }
        // Other lists: one round trip reads their counters (lanes of the first
        // wavefront, atomic reads at the same coherence point as the claims)
        // and picks the first, in queue order after this one, with items left.
        // Every claim advances a counter, so the loop ends; the bound is a
        // second guarantee.
        for (int round = 0; round <= plan[H_N_TAIL] + kXcdQueues; ++round) {
          if (threadIdx.x < 64) {
            const int l = threadIdx.x;
            const int q = home + 1 + l < kXcdQueues ? home + 1 + l : home + 1 + l - kXcdQueues;
            bool left = false;
            if (l < kXcdQueues - 1)
              left = int(__hip_atomic_fetch_add(ctr + q * kCounterWords, 0u, __ATOMIC_RELAXED,
                                                __HIP_MEMORY_SCOPE_AGENT)) < tab[kXcdQueues + q];
            const uint64_t m = __ballot(left);
            if (l == 0) {
              const int f = m ? __builtin_ctzll(m) : -1;
              claim_sh = f < 0 ? -1 : (home + 1 + f) % kXcdQueues;
            }
          }
          __syncthreads();
          const int q = __builtin_amdgcn_readfirstlane(claim_sh);
          __syncthreads();
          if (q < 0) break;
          const int c = claim(q);
          if (c < tab[kXcdQueues + q]) run(q, c);
        }
        uint32_t* done = ctr + kXcdQueues * kCounterWords;
        if (threadIdx.x == 0 &&
            __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 ==
                uint32_t(plan[H_N_WILD])) {
          // every other wildcard workgroup has made its last claims
          for (int q = 0; q <= kXcdQueues; ++q)
            __hip_atomic_exchange(ctr + q * kCounterWords, 0u, __ATOMIC_RELAXED,
                                  __HIP_MEMORY_SCOPE_AGENT);
        }
        return;
      }
    }
    if (ti < n_shared) {
      const int32_t* it = plan + plan[H_SHARED_OFF] + ti * kSharedWords;
      if (it[S_NROWS] > kTileRows - 32) tile_item<D, kTileSub, BITS, true, true>(it, g, poff, a, sm);
      else tile_item<D, kTileSub, BITS, true, false>(it, g, poff, a, sm);
      return;
    }
    if (ti < n_tile) {
      const int32_t* it = plan + plan[H_TILE_OFF] + (ti - n_shared) * kItemWords;
      // every wavefront has rows: the plain path; otherwise idle ones skip
      // compute, and a few-row sequence's private keys are streamed
      if (it[I_NROWS] > kTileRows - 32) tile_item<D, kTileSub, BITS, false, true>(it, g, poff, a, sm);
      else if (it[I_FLAGS] & kItemStream) tile_item<D, kTileSub, BITS, false, false, true>(it, g, poff, a, sm);
      else tile_item<D, kTileSub, BITS, false, false>(it, g, poff, a, sm);
      return;
    }
  }
  if constexpr ((MIX & 6) != 0) {
    __shared__ JoinStat stat8[4][2][16];
    if (ti >= n_tile) {
      // a quad of row templates, one per wavefront
      const int32_t* it =
          plan + plan[H_ROW_OFF] + (ti - n_tile + (threadIdx.x >> 6)) * kItemWords;
      if constexpr ((MIX & 4) != 0) {
        if (it[I_NROWS] > 16) {
          if constexpr (kQuantised) {
            auto& join = *reinterpret_cast<JoinSmem<D, 2>*>(lds8);
            if (it[I_FLAGS] & kItemTwice) row_item8<D, 2, BITS, false, true>(it, g, poff, a, join, stat8);
            else row_item8<D, 2, BITS, false, false>(it, g, poff, a, join, stat8);
          } else {
            row_item<D, 2>(it, g, poff, a);
          }
          return;
        }
      }
      if constexpr (kQuantised) {
        auto& join = *reinterpret_cast<JoinSmem<D, 1>*>(lds8);
        if constexpr ((MIX & 4) != 0) {
          if (it[I_FLAGS] & kItemTwice) {
            row_item8<D, 1, BITS, false, true>(it, g, poff, a, join, stat8);
            return;
          }
        }
        row_item8<D, 1, BITS, MIX == 2 && !(BITS == 4 && D == 64), false>(it, g, poff, a, join, stat8);
      } else {
        row_item<D, 1>(it, g, poff, a);
      }
    }
  }
}

}  // namespace

// Launches a plan's items over a cache of BITS bits a value.  Each cache's kernels are
// instantiated by a source file of their own: they compile side by side.
template <int BITS>
int launch_items(const AttnArgs& a, int32_t d, int32_t mix, int32_t grid, hipStream_t stream,
                 hipEvent_t ev_start, hipEvent_t ev_stop) {
#define PA_LAUNCH(DD, MM)                                                                        \
  hipExtLaunchKernelGGL((attn_bf16_kernel<DD, MM, BITS>), dim3(grid), dim3(256), 0, stream,      \
                        ev_start, ev_stop, 0, a)
#define PA_LAUNCH_D(DD)                      \
  switch (mix) {                             \
    case 1: PA_LAUNCH(DD, 1); break;         \
    case 2: PA_LAUNCH(DD, 2); break;         \
    case 6: PA_LAUNCH(DD, 6); break;         \
    case 9: PA_LAUNCH(DD, 9); break;         \
    case 15: PA_LAUNCH(DD, 15); break;       \
    default: PA_LAUNCH(DD, 7); break;        \
  }
  if (d == 128) {
    PA_LAUNCH_D(128);
  } else {
    PA_LAUNCH_D(64);
  }
#undef PA_LAUNCH_D
#undef PA_LAUNCH
  return static_cast<int>(hipGetLastError());
}

}  // namespace dev
}  // namespace pa
