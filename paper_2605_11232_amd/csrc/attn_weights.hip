// Attention weights of cached keys: for each sequence r, kv-head h and key t,
//   W[r][h][t] = sum over the sequence's rows i and the heads g of h's group that see t
//                of exp(scale * q_ig . k_t - lse_ig),
// the keys' column sums of the probabilities that the attention call formed, from its
// queries and log-sum-exps (a row's sum need not be found again).  Only keys are read, not
// values: half the cache's bytes.
//
// S = Q K^T on 32x32x16 MFMA with a key in each lane, so a lane adds its key's
// probabilities over 16 rows without looking at other lanes; the two lane halves (other
// rows) are added once at the end.  A workgroup owns its keys and goes over all rows of the
// sequence: no atomics, one order of the sums, and keys are read once.  Three ways: many
// rows that a workgroup's wavefronts share; many rows of few keys, which they divide; few
// rows, which stay in registers.
#include <type_traits>

#include "device_common.h"

namespace pa {
namespace dev {
namespace {

struct WeightArgs {
  const __bf16* q;
  const float* lse;
  const uint8_t* kc;
  const uint8_t* scales;  // 4 bits
  const int32_t* bt;
  const int32_t* seq_lens;
  const int32_t* cu;
  float* w;
  int64_t w_stride;
  int32_t max_blocks, num_blocks, total_q, hq, hkv;
  int32_t chunks;  // workgroups of a (sequence, kv-head)
  int32_t heads;   // (sequence, kv-head) pairs, where all their first workgroups come first, or 0
  int32_t range;   // few rows: keys of a wavefront at a time
  int32_t n_seqs;
  int32_t limit;   // few rows: sequences of more rows are left to the other kernels, which take
  bool longs;      // only those then
  float scale_log2;
  bool add;
};

constexpr int kRows = 32;  // rows at a time
// Wavefronts wanted where rows are few (64 requests of 2048-8192 keys: 4096 137 us, 8192 124,
// 16384 122).
constexpr int kFewWaves = 16384;

// LDS: two tiles of rows, 16-byte unit p of row r at unit p ^ (r & 7), so that eight
// neighbouring lanes (rows) read distinct banks; the rows' log-sum-exps (times log2 e) and
// positions (a row that does not count: -1, it sees no key); the position up to which all of
// the tile's rows see keys.
template <int D>
struct RowSmem {
  __bf16 q[2][kRows * D];
  float lse[2][kRows];
  int pos[2][kRows];
  int seen[2];
};

// A sequence's rows and keys, as the kernels see them.
struct SeqRows {
  int qs, rows, base, keys;  // first row's token, rows of a kv-head, its position, keys with weights
};
__device__ __forceinline__ SeqRows rows_of(const WeightArgs& a, int r) {
  const int qs = a.cu[r], all = a.cu[r + 1] - qs, L = a.seq_lens[r];
  const int n = min(a.cu[r + 1], a.total_q) - qs;
  if (qs < 0 || n <= 0 || L < all) return {0, 0, 0, 0};
  return {qs, n * (a.hq / a.hkv), L - all, int(min(int64_t(L), min(a.w_stride, int64_t(a.max_blocks) * kBlock)))};
}
// The n-th sequence of more than a.limit rows, or -1.
__device__ __forceinline__ int nth_long(const WeightArgs& a, int n) {
  const int lane = threadIdx.x & 63;
  for (int r0 = 0; r0 < a.n_seqs; r0 += 64) {
    const int r = r0 + lane;
    uint64_t m = __ballot(r < a.n_seqs && rows_of(a, min(r, a.n_seqs - 1)).rows > a.limit);
    const int c = __popcll(m);
    if (n < c) {
      for (; n > 0; --n) m &= m - 1;
      return r0 + __builtin_ctzll(m);
    }
    n -= c;
  }
  return -1;
}
__device__ __forceinline__ bool counts(float lse) { return fabsf(lse) < __builtin_huge_valf(); }

// Eight e2m1 codes times the power of two of a scale byte (255: NaN), as bf16 (exact).
__device__ __forceinline__ bf16x8 bf16_of_codes(uint32_t v, uint32_t byte) {
  const float f = __uint_as_float(byte << 23);
  return as_bf16x8(u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, f, 0)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, f, 1)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, f, 2)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, f, 3))});
}

// A lane's part of key `o` of (block, kv-head) b, half hh, as the product's operand: natural
// k-steps over a bf16 cache; over a 4-bit one dims (D/2) hh + 8 ks, which lie together.
template <int D, int BITS>
struct KeyRegs {
  static constexpr int KS = D / 16;
  u32x4 x[BITS == 16 ? KS : D / 64];
  uint32_t sc[D / 64];
  __device__ __forceinline__ void load(const WeightArgs& a, int64_t b, int o, int hh) {
    if constexpr (BITS == 16) {
      const __bf16* p = reinterpret_cast<const __bf16*>(a.kc) + b * (kBlock * D) + key_slot_pos(o) * kKeyGroup + 8 * hh;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        x[ks] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + (ks / 2) * (kBlock * kKeyGroup) + 16 * (ks % 2)));
    } else {
      const uint8_t* p = a.kc + b * (kBlock * D / 2) + o * (D / 2) + hh * (D / 4);
      const uint8_t* s = a.scales + b * ((D / 32 + 1) * kBlock) + hh * (D / 64) * kBlock + o;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 16 * i));
        sc[i] = s[i * kBlock];
      }
    }
  }
  __device__ __forceinline__ bf16x8 operand(int ks) const {
    if constexpr (BITS == 16) {
      return as_bf16x8(x[ks]);
    } else {
      return bf16_of_codes(x[ks / 4][ks % 4], sc[ks / 4]);
    }
  }
  // 16-byte unit of a row of q that k-step ks multiplies.
  __device__ static __forceinline__ int unit(int ks, int hh) { return BITS == 16 ? 2 * ks + hh : hh * KS + ks; }
};

// Many rows: a workgroup's four wavefronts share each tile of 32 rows through LDS; 64 keys
// a wavefront, which stay in registers.  Bound by issue: a step's products and, a score, a
// fused multiply-add, an exponential and an addition (16 sequences of 4096-12000 4-bit keys
// under 64 rows of 28/4 heads: 76 us, of which the vector units issue for 45 and the matrix
// units work for 25, 2.1 wavefronts a SIMD, 2.6 rounds of workgroups).  Before the rows' loads
// went out without waits between they took 153; tiles of 64 rows 97 against 92 at the time,
// two or eight wavefronts a workgroup, or two a SIMD, 117.  One key tile's probabilities between
// the other's products, in one wavefront, take 123 (32 registers spilled), at two wavefronts a
// SIMD 102: products of a single accumulator wait for each other.
template <int D, int BITS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void attn_weights_kernel(WeightArgs a) {
  constexpr int KT = 2;               // 32-key tiles of a wavefront
  constexpr int KS = D / 16;          // k-steps
  constexpr int UR = D / 8;           // 16-byte units of a row
  constexpr int NL = kRows * UR / 256;  // units of a thread
  constexpr int kChunk = 4 * 32 * KT;
  __shared__ __align__(16) RowSmem<D> sm;
  const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, hh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  int x = blockIdx.x / a.chunks, first_chunk = blockIdx.x - x * a.chunks;
  if (a.heads > 0) {
    first_chunk = blockIdx.x / a.heads;
    x = (blockIdx.x - first_chunk * a.heads + first_chunk) % a.heads;
  }
  int r = x / a.hkv;
  const int g = x - r * a.hkv;
  if (a.longs) {
    r = __builtin_amdgcn_readfirstlane(nth_long(a, r));
    if (r < 0) return;
  }
  const SeqRows sr = rows_of(a, r);
  const int rows = sr.rows, L = sr.keys, G = a.hq / a.hkv;
  if (rows == 0) return;
  const float c = a.scale_log2;
  const int32_t* bt = a.bt + (int64_t)r * a.max_blocks;
  // a tile's rows as queries and heads, and how far that is in (token, head) rows
  const int step_q = kRows / G, step_h = kRows - step_q * G, step_row = step_q * a.hq + step_h;

  // Rows of the next tile that this thread copies: units 256 i + tid, log-sum-exp tid.
  // All of a stage's loads are issued at once; whether a row counts is looked at when it is
  // stored.
  u32x4 raw[NL];
  float raw_z[NL], raw_lse = 0.f;
  int raw_pos = 0;
  const __bf16* const q0 = a.q + ((int64_t)sr.qs * a.hq + g * G) * D + 8 * (tid % UR);
  const float* const z0 = a.lse + (int64_t)sr.qs * a.hq + g * G;
  int row[NL], head[NL], row_z = 0, head_z = 0, pos_z = 0;
  auto seek_rows = [&](int r0) {
    auto of = [&](int rho, int& rw, int& h) {
      const int qi = rho / G;
      h = rho - qi * G, rw = qi * a.hq + h;
      return sr.base + qi;
    };
#pragma unroll
    for (int i = 0; i < NL; ++i) of(r0 + (256 * i + tid) / UR, row[i], head[i]);
    pos_z = of(r0 + tid, row_z, head_z);
  };
  // one tile on; whether that passes one more query
  auto advance = [&](int& rw, int& h) {
    rw += step_row, h += step_h;
    const bool next = h >= G;
    if (next) h -= G, rw += a.hq - G;
    return next;
  };
  auto load_rows = [&](int r0) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const bool in = r0 + (256 * i + tid) / UR < rows;
      const int at = in ? row[i] : 0;
      raw[i] = ld16(q0 + (int64_t)at * D);
      raw_z[i] = in ? z0[at] : __builtin_huge_valf();
      advance(row[i], head[i]);
    }
    if (tid < kRows) {
      const bool in = r0 + tid < rows;
      raw_lse = in ? z0[row_z] : __builtin_huge_valf();
      raw_pos = in ? pos_z : -1;
      pos_z += step_q + advance(row_z, head_z);
    }
  };
  auto store_rows = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = 256 * i + tid, lr = u / UR, p = u % UR;
      st16(&sm.q[buf][8 * (lr * UR + (p ^ (lr & 7)))], counts(raw_z[i]) ? raw[i] : zero16());
    }
    if (tid < kRows) {
      const bool ok = counts(raw_lse);
      sm.lse[buf][tid] = ok ? raw_lse * kLog2e : __builtin_huge_valf();
      sm.pos[buf][tid] = ok ? raw_pos : -1;
      const bool all = __ballot(!ok) == 0;
      if (tid == 0) sm.seen[buf] = all ? raw_pos : -1;
    }
  };

  for (int64_t chunk = first_chunk; chunk * kChunk < L; chunk += a.chunks) {
    const int key0 = int(chunk) * kChunk;
    // rows from the first that sees one of the chunk's keys on
    const int row_first = min(max(0, key0 - sr.base), rows / G) * G / kRows * kRows;
    seek_rows(row_first);
    load_rows(row_first);
    bf16x8 k[KT][KS];
    int key[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      key[t] = key0 + (w * KT + t) * 32 + j;
      const int kk = min(key[t], L - 1);
      KeyRegs<D, BITS> raw_k;
      raw_k.load(a, (int64_t)clamp_block(bt[kk / kBlock], a.num_blocks) * a.hkv + g, kk % kBlock, hh);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k[t][ks] = raw_k.operand(ks);
    }
    float sum[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) sum[t] = 0.f;
    const int last_key = min(key0 + (w * KT + KT) * 32, L) - 1;  // of this wavefront
    int buf = 0;
    store_rows(0);
    __syncthreads();
    for (int r0 = row_first; r0 < rows; r0 += kRows, buf ^= 1) {
      const bool more = r0 + kRows < rows;
      if (more) load_rows(r0 + kRows);
      f32x16 s[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
      // reads of the rows go three k-steps ahead of the products
      u32x4 qx[3];
      auto q_of = [&](int ks) {
        const int p = KeyRegs<D, BITS>::unit(ks, hh);
        return ld16(&sm.q[buf][8 * (j * UR + (p ^ (j & 7)))]);
      };
#pragma unroll
      for (int i = 0; i < 3; ++i) qx[i] = q_of(i);
      __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 q = as_bf16x8(qx[ks % 3]);
        if (ks + 3 < KS) {
          qx[ks % 3] = q_of(ks + 3);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
#pragma unroll
        for (int t = 0; t < KT; ++t) s[t] = mfma32(q, k[t][ks], s[t]);
        __builtin_amdgcn_sched_group_barrier(0x008, KT, 0);
      }
      // a row does not see all keys: positions are looked at, so that an infinite key is
      // multiplied with a row that does not count to no effect
      auto add = [&](auto masked) {
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 z = *reinterpret_cast<const f32x4*>(&sm.lse[buf][8 * q4 + 4 * hh]);
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float p = fast_exp2(fmaf(s[t][4 * q4 + e], c, -z[e]));
              if constexpr (decltype(masked)::value) p = key[t] <= sm.pos[buf][8 * q4 + 4 * hh + e] ? p : 0.f;
              sum[t] += p;
            }
        }
      };
      if (__builtin_amdgcn_readfirstlane(sm.seen[buf]) < last_key) add(std::true_type{});
      else add(std::false_type{});
      if (more) store_rows(buf ^ 1);
      __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      sum[t] += wave_xor(sum[t], 32);
      if (hh == 0 && key[t] < L) {
        float* p = a.w + ((int64_t)r * a.hkv + g) * a.w_stride + key[t];
        *p = a.add ? *p + sum[t] : sum[t];
      }
    }
  }
}

// Many rows of few keys, where workgroups of 256 keys would leave most of the chip idle: a
// workgroup owns 32 KT keys, each of its NW wavefronts goes over every NW-th tile of the rows,
// in LDS of its own without barriers, and the wavefronts' sums are added in order.  8
// wavefronts on 64 keys, or 16 on 32 where those are no more workgroups than CUs (12 on 64
// are 5 to 20 % slower than 8).  Bound by latency and by the rows' way through LDS, which 64
// keys share instead of 256 (one sequence of 700 keys under 1680 rows of 4 kv-heads 10.9 us,
// 53.8 by the kernel above; in which two or three groups of wavefronts that divide the rows
// take as long as one up to 256 workgroups, since their barriers keep them in step).
template <int D>
struct WaveRows {
  __bf16 q[kRows * D];
  float lse[kRows];
  int pos[kRows];
};
template <int D, int BITS, int NW, int KT>
__global__ __launch_bounds__(64 * NW) void attn_weights_split_kernel(WeightArgs a) {
  constexpr int KS = D / 16, UR = D / 8, kChunk = 32 * KT;
  constexpr int NL = kRows * UR / 64;  // 16-byte units of a lane
  __shared__ __align__(16) WaveRows<D> sm[NW];
  __shared__ float part[NW][kChunk];
  const int lane = threadIdx.x & 63, j = lane & 31, hh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int x = blockIdx.x / a.chunks, first_chunk = blockIdx.x - x * a.chunks;
  int r = x / a.hkv;
  const int g = x - r * a.hkv;
  if (a.longs) {
    r = __builtin_amdgcn_readfirstlane(nth_long(a, r));
    if (r < 0) return;
  }
  const SeqRows sr = rows_of(a, r);
  const int rows = sr.rows, L = sr.keys, G = a.hq / a.hkv;
  if (rows == 0) return;
  const float c = a.scale_log2;
  const int32_t* bt = a.bt + (int64_t)r * a.max_blocks;
  const __bf16* const q0 = a.q + ((int64_t)sr.qs * a.hq + g * G) * D + 8 * (lane % UR);
  const float* const z0 = a.lse + (int64_t)sr.qs * a.hq + g * G;
  WaveRows<D>& mine = sm[w];
  u32x4 raw[NL];
  float raw_lse = 0.f;
  int raw_pos = 0;
  auto load_rows = [&](int r0) {
    const int rho = min(r0 + j, rows - 1), qi = rho / G, at = qi * a.hq + rho - qi * G;
#pragma unroll
    for (int i = 0; i < NL; ++i) raw[i] = ld16(q0 + (int64_t)__shfl(at, (64 * i + lane) / UR, 64) * D);
    raw_lse = z0[at];
    raw_pos = r0 + j < rows ? sr.base + qi : -1;
  };
  for (int64_t chunk = first_chunk; chunk * kChunk < L; chunk += a.chunks) {
    const int key0 = int(chunk) * kChunk, last_key = min(key0 + kChunk, L) - 1;
    int r0 = min(max(0, key0 - sr.base), rows / G) * G / kRows * kRows + w * kRows;
    if (r0 < rows) load_rows(r0);
    bf16x8 k[KT][KS];
    float sum[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const int kk = min(key0 + 32 * t + j, L - 1);
      KeyRegs<D, BITS> raw_k;
      raw_k.load(a, (int64_t)clamp_block(bt[kk / kBlock], a.num_blocks) * a.hkv + g, kk % kBlock, hh);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k[t][ks] = raw_k.operand(ks);
      sum[t] = 0.f;
    }
    for (; r0 < rows; r0 += NW * kRows) {
      wave_lds_order();
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int u = 64 * i + lane, lr = u / UR, p = u % UR;
        st16(&mine.q[8 * (lr * UR + (p ^ (lr & 7)))], raw[i]);
      }
      const bool ok = raw_pos >= 0 && counts(raw_lse);
      const bool all = __ballot(!ok) == 0;
      const int seen = all ? __builtin_amdgcn_readfirstlane(raw_pos) : -1;
      if (hh == 0) {
        mine.lse[j] = ok ? raw_lse * kLog2e : __builtin_huge_valf();
        mine.pos[j] = ok ? raw_pos : -1;
      }
      wave_lds_order();
      if (r0 + NW * kRows < rows) load_rows(r0 + NW * kRows);
      f32x16 s[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int p = KeyRegs<D, BITS>::unit(ks, hh);
        const bf16x8 q = as_bf16x8(ld16(&mine.q[8 * (j * UR + (p ^ (j & 7)))]));
#pragma unroll
        for (int t = 0; t < KT; ++t) s[t] = mfma32(q, k[t][ks], s[t]);
      }
      auto add = [&](auto masked) {
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4 z = *reinterpret_cast<const f32x4*>(&mine.lse[8 * q4 + 4 * hh]);
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float p = fast_exp2(fmaf(s[t][4 * q4 + e], c, -z[e]));
              if constexpr (decltype(masked)::value)
                p = key0 + 32 * t + j <= mine.pos[8 * q4 + 4 * hh + e] ? p : 0.f;
              sum[t] += p;
            }
        }
      };
      if (seen < last_key) add(std::true_type{});
      else add(std::false_type{});
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      sum[t] += wave_xor(sum[t], 32);
      if (hh == 0) part[w][32 * t + j] = sum[t];
    }
    __syncthreads();
    const int key = key0 + threadIdx.x;
    if (threadIdx.x < kChunk && key < L) {
      float total = part[0][threadIdx.x];
#pragma unroll
      for (int v = 1; v < NW; ++v) total += part[v][threadIdx.x];
      float* p = a.w + ((int64_t)r * a.hkv + g) * a.w_stride + key;
      *p = a.add ? *p + total : total;
    }
    __syncthreads();
  }
}

// A lane's part of a key (16x16x32 MFMA: lane (j, g4) of key j), so that the four lanes of a
// key read the 64 bytes that lie together: dims 32 ks + 8 g4 over a bf16 cache, (D/4) g4 +
// 8 ks over a 4-bit one.
template <int D, int BITS>
struct KeyRegs16 {
  static constexpr int KS = D / 32;
  typedef uint32_t words __attribute__((ext_vector_type(BITS == 16 ? 4 : D / 32)));
  words x[BITS == 16 ? KS : 1];
  uint32_t sc;
  __device__ __forceinline__ void load(const WeightArgs& a, int64_t b, int o, int g4) {
    if constexpr (BITS == 16) {
      const __bf16* p = reinterpret_cast<const __bf16*>(a.kc) + b * (kBlock * D) + key_slot_pos(o) * kKeyGroup + 8 * g4;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        x[ks] = __builtin_nontemporal_load(reinterpret_cast<const words*>(p + ks * (kBlock * kKeyGroup)));
    } else {
      x[0] = __builtin_nontemporal_load(reinterpret_cast<const words*>(a.kc + b * (kBlock * D / 2) + o * (D / 2) + g4 * (D / 8)));
      sc = a.scales[b * ((D / 32 + 1) * kBlock) + (D == 128 ? g4 : g4 >> 1) * kBlock + o];
    }
  }
  __device__ __forceinline__ bf16x8 operand(int ks) const {
    if constexpr (BITS == 16) return as_bf16x8(x[ks]);
    else return bf16_of_codes(x[0][ks], sc);
  }
  __device__ static __forceinline__ int unit(int ks, int g4) { return BITS == 16 ? 4 * ks + g4 : g4 * KS + ks; }
};

// Few rows (a decode or verification step): the keys are what takes time.  A wavefront
// holds 16 NR rows in registers and goes over up to 64 blocks of keys, 32 keys ahead of those
// that it multiplies; nothing is shared.  Sequences of more rows go over their keys once for
// each 16 NR.  Bound by the keys' bytes: a decode step of 64 requests of 2048-8192 bf16 keys,
// 32/8 heads, 121 us, 5.8 TB/s (on 32x32x16 products, whose lanes' loads of 16 bytes each lie
// 64 apart, 149).
template <int D, int BITS, int NR>
__global__ __launch_bounds__(256) void attn_weights_few_kernel(WeightArgs a) {
  using Keys = KeyRegs16<D, BITS>;
  constexpr int KS = Keys::KS;
  const int lane = threadIdx.x & 63, j = lane & 15, g4 = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int x = blockIdx.x / a.chunks;
  const int r = x / a.hkv, g = x - r * a.hkv;
  const SeqRows sr = rows_of(a, r);
  const int G = a.hq / a.hkv, L = sr.keys;
  const int32_t* bt = a.bt + (int64_t)r * a.max_blocks;
  float* wp = a.w + ((int64_t)r * a.hkv + g) * a.w_stride;
  const float c = a.scale_log2;
  for (int64_t i = (blockIdx.x - x * a.chunks) * 4 + w; i * a.range < L && sr.rows > 0 && sr.rows <= a.limit; i += 4 * a.chunks) {
    const int k0 = int(i) * a.range, k1 = min(k0 + a.range, L);
    BlockSpan span;
    span.init(bt, a.max_blocks, k0 / kBlock);
    for (int r0 = 0; r0 < sr.rows; r0 += 16 * NR) {
      int seen = sr.base + r0 / G;  // up to here all rows see keys
      bf16x8 q[NR][KS];
      f32x4 z[NR];
      int pos[NR][4];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        // row j, its query as the product's operand, its log-sum-exp and position
        const int lr = r0 + 16 * n + j, rho = min(lr, sr.rows - 1), qi = rho / G;
        const int64_t row = (int64_t)(sr.qs + qi) * a.hq + g * G + (rho - qi * G);
        const float lse = a.lse[row];
        const bool ok = lr < sr.rows && counts(lse);
        const float my_z = ok ? lse * kLog2e : __builtin_huge_valf();
        const int my_pos = ok ? sr.base + qi : -1;  // -1: it sees no key
        if (__ballot(!ok) != 0) seen = -1;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const u32x4 v = ld16(a.q + row * D + 8 * Keys::unit(ks, g4));
          q[n][ks] = as_bf16x8(ok ? v : zero16());
        }
        // of rows 4 g4 + e, which the lane's scores belong to
#pragma unroll
        for (int e = 0; e < 4; ++e) z[n][e] = __shfl(my_z, 4 * g4 + e, 64), pos[n][e] = __shfl(my_pos, 4 * g4 + e, 64);
      }
      Keys k[2][2];
      auto load = [&](int t0, int s) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int key = min(t0 + 16 * t + j, k1 - 1);
          const int id = span.get(min(t0 / kBlock + t, (k1 - 1) / kBlock));
          k[s][t].load(a, (int64_t)clamp_block(id, a.num_blocks) * a.hkv + g, key % kBlock, g4);
        }
      };
      auto step = [&](int t0, auto b) {
        constexpr int cur = decltype(b)::value;
        if (t0 + 32 < k1) load(t0 + 32, 1 - cur);
        const bool masked = t0 + 31 > seen;
        float sum[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4 s[NR];
#pragma unroll
          for (int n = 0; n < NR; ++n) s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const bf16x8 x = k[cur][t].operand(ks);
#pragma unroll
            for (int n = 0; n < NR; ++n) s[n] = mfma16(q[n][ks], x, s[n]);
          }
          sum[t] = 0.f;
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float p = fast_exp2(fmaf(s[n][e], c, -z[n][e]));
              if (masked) p = t0 + 16 * t + j <= pos[n][e] ? p : 0.f;
              sum[t] += p;
            }
          sum[t] += wave_xor(sum[t], 16);
          sum[t] += wave_xor(sum[t], 32);
        }
        const int key = t0 + lane;
        const float s = lane < 16 ? sum[0] : sum[1];
        if (lane < 32 && key < k1) wp[key] = a.add || r0 > 0 ? wp[key] + s : s;
      };
      load(k0, 0);
      for (int t0 = k0; t0 < k1; t0 += 64) {
        step(t0, std::integral_constant<int, 0>{});
        if (t0 + 32 < k1) step(t0 + 32, std::integral_constant<int, 1>{});
      }
    }
  }
}

}  // namespace

// The kernels for many rows: n_seqs sequences at most, of which the host reckons with `likely`
// of `rows` rows a kv-head.
void launch_many(WeightArgs a, int64_t n_seqs, int64_t rows, int64_t likely, int64_t keys, int32_t d,
                 int32_t bits, hipStream_t stream) {
  const int64_t heads = n_seqs * a.hkv;
  int64_t chunk = 256;  // keys of a workgroup
  // Where workgroups of 256 keys are few, of 64 keys, and of 32 where those are no more than
  // CUs.  In units of 10 ns the first, up to one a CU, take 360 + 95 for each 32 rows, a round
  // of the second 500 + 20, at head_dim 64 300 + 12 (4 or 8 kv-heads of 128, bf16; workgroups
  // of 256 keys: us by them, by 64 keys and by 32): 1200 rows 16: 41 11.3 9.1, 64: 42 17.1 24,
  // 192: 44 39 55, 256: 45 48 70; 120 rows 64: 7.6 5.6 8.1, 128: 7.8 9.1 13.7; 10500 rows
  // 24: 322 62 50, 96: 327 119 140, 192: 327 194 265, 384: 339 353 507.
  const int64_t steps = (rows + kRows - 1) / kRows, n64 = likely * a.hkv * ((keys + 63) / 64);
  const bool split = n64 <= 2048 && max(n64, int64_t(256)) * (d == 64 ? 300 + 12 * steps : 500 + 20 * steps) <
                                        256 * (360 + 95 * steps);
  const bool fine = split && likely * a.hkv * ((keys + 31) / 32) <= 256;
  if (split) chunk = fine ? 32 : 64;
  // few workgroups without keys where the array is wider than the sequences are long
  const int64_t chunks = min((keys + chunk - 1) / chunk, max(int64_t(1), 32768 / heads));
  a.chunks = int32_t(chunks);
  // A prompt's first keys have the most rows: where new tokens are many beside the keys, all
  // sequences' first workgroups go first, and the next ones' XCDs are others.  Else a sequence's
  // go together, whose rows stay in the L2 caches.  us one way and the other: 33 prompts of
  // 1167-1320 tokens, 28/4 heads, 450 and 341, 60 of 100-2000 on the 4-bit cache 1231 and 579,
  // 12 of 1000-1500 on 3000-5000 keys, 32/8 heads, 738 and 669; 16 of 64 tokens on 4096-12000
  // 80 and 85, 20 of 200-600 on 1000-2000 180 and 205.
  if (!split && 6 * rows >= keys * (a.hq / a.hkv)) a.heads = int32_t(heads);
  const dim3 grid(unsigned(heads * chunks));
#define PA_W(N, ...) hipLaunchKernelGGL((__VA_ARGS__), grid, dim3(N), 0, stream, a)
#define PA_W_MANY(DD, BB)                                              \
  {                                                                    \
    if (fine) PA_W(1024, attn_weights_split_kernel<DD, BB, 16, 1>);    \
    else if (split) PA_W(512, attn_weights_split_kernel<DD, BB, 8, 2>); \
    else PA_W(256, attn_weights_kernel<DD, BB>);                       \
  }
#define PA_W_FEW(DD, BB)                                                               \
  {                                                                                    \
    if (BB == 16 && rows > 32) PA_W(256, attn_weights_few_kernel<DD, 16, 4>);          \
    else if (rows > 16) PA_W(256, attn_weights_few_kernel<DD, BB, 2>);                 \
    else PA_W(256, attn_weights_few_kernel<DD, BB, 1>);                                \
  }
#define PA_W_BITS(M)                 \
  if (d == 128 && bits == 16) M(128, 16) \
  else if (d == 128) M(128, 4)       \
  else if (bits == 16) M(64, 16)     \
  else M(64, 4)
  PA_W_BITS(PA_W_MANY)
}

int launch_attn_weights(const void* q, const float* lse, const void* kc, const uint8_t* scales,
                        int32_t num_blocks, const int32_t* bt, int32_t max_blocks,
                        const int32_t* seq_lens, const int32_t* cu, int32_t n_seqs, int32_t total_q,
                        int32_t hq, int32_t hkv, int32_t d, int32_t bits, float scale, float* w,
                        int64_t w_stride, bool add, hipStream_t stream) {
  WeightArgs a{static_cast<const __bf16*>(q), lse, static_cast<const uint8_t*>(kc), scales, bt, seq_lens,
               cu, w, w_stride, max_blocks, num_blocks, total_q, hq, hkv, 0, 0, 0, n_seqs, INT32_MAX, false,
               scale * kLog2e, add};
  const int64_t heads = int64_t(n_seqs) * hkv, keys = min(w_stride, int64_t(max_blocks) * kBlock);
  // Rows of a kv-head, of the average sequence.  32 sequences of 2048-8192 keys, 32/8 heads:
  // bf16 16 rows 61 us (through LDS 94), 32 rows 67 (96), 64 rows 90 (103), 4 bits 30 (48), 42
  // (49), 76 (59).
  const int64_t rows = (int64_t(total_q) * (hq / hkv) + n_seqs - 1) / n_seqs;
  const bool many = rows > (bits == 16 ? 64 : 32);
  if (heads > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
  if (many) {
    launch_many(a, n_seqs, rows, n_seqs, keys, d, bits, stream);
    return static_cast<int>(hipGetLastError());
  }
  // wavefronts of as many keys as leave enough of them to fill the chip
  a.range = int32_t(max(int64_t(1), min(int64_t(32), keys * heads / (32 * kFewWaves)))) * 32;
  const int64_t chunks = min((keys + 4 * a.range - 1) / (4 * a.range), max(int64_t(1), 32768 / heads));
  a.chunks = int32_t(chunks);
  // Prompts among requests of few rows: a launch of its own for sequences of more than `limit`
  // rows, as many as there can be (us with one launch and two: 95 requests of 500-1500 keys,
  // 32/8 heads of 64 dims on the 4-bit cache, and prompts of 512 and 100 tokens 166 and 46, 199
  // of 200-1000 and one of 1000 804 and 97, 64 of 2000-6000 and one of 512 341 and 175; the
  // other way, 186 of 500-1500 4-bit keys and 8 of 150 tokens 129 and 176).  The host does not
  // have the lengths: a total that divides by the sequences is taken for the same number of rows
  // in each, and each sequence for one of a row or more.  Where that is not so the prompts stay
  // with the others, in one launch, to the same formula in more time.
  // The limit, one prompt among 96 requests of 500-1500 keys, 32/8 heads of 128, one launch and
  // two: bf16 80 rows a kv-head 39 and 45, 112 41 and 46, 160 48 and 47, 288 71 and 51, 4 bits
  // 48 rows 22.7 and 27.8, 80 22.8 and 28.9, 160 32 and 31; among 64 of 2000-6000: bf16 160
  // 133 and 108, 4 bits 80 43 and 46, 112 53 and 47.
  // Prompts reckoned with, 1, 2 and 4: two of 300 tokens among 128 requests of 2000-6000 bf16
  // keys 344, 261 and 261, four among 190 of 500-1500 166, 166 and 137, one of 136 among 96 of
  // these 49, 48 and 60.
  const int64_t G = hq / hkv, limit = bits == 16 ? 128 : 64, longs = min(int64_t(n_seqs), total_q * G / (limit + 1));
  const bool mixed = total_q % n_seqs != 0 && (int64_t(total_q) - n_seqs + 1) * G > limit;
  if (mixed) a.limit = int32_t(limit);
  const dim3 grid(unsigned(heads * chunks));
  PA_W_BITS(PA_W_FEW)
  if (mixed) {
    a.longs = true;
    const int64_t likely = min(longs, int64_t(2));
    launch_many(a, longs, (int64_t(total_q) - n_seqs + 1) * G / likely, likely, keys, d, bits, stream);
  }
#undef PA_W_BITS
#undef PA_W_FEW
#undef PA_W_MANY
#undef PA_W
  return static_cast<int>(hipGetLastError());
}

}  // namespace dev
}  // namespace pa
