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
// sequence: no atomics, one order of the sums, and keys are read once.
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
  int32_t max_blocks, num_blocks, total_q, hq, hkv, chunks;
  float scale_log2;
  bool add;
};

constexpr int kRows = 32;  // rows at a time

// LDS: two tiles of rows, 16-byte unit p of row r at unit p ^ (r & 7), so that eight
// neighbouring lanes (rows) read distinct banks; the rows' log-sum-exps (times log2 e; a row
// that does not count: infinity) and positions.
template <int D>
struct RowSmem {
  __bf16 q[2][kRows * D];
  float lse[2][kRows];
  int pos[2][kRows];
};

// KT: 32-key tiles of a wavefront.
template <int D, int BITS, int KT>
__global__ __launch_bounds__(256) void attn_weights_kernel(WeightArgs a) {
  constexpr int KS = D / 16;          // k-steps
  constexpr int UR = D / 8;           // 16-byte units of a row
  constexpr int NL = kRows * UR / 256;  // units of a thread
  constexpr int kChunk = 4 * 32 * KT;
  __shared__ __align__(16) RowSmem<D> sm;
  const int tid = threadIdx.x, lane = tid & 63, j = lane & 31, hh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int x = blockIdx.x / a.chunks, first_chunk = blockIdx.x - x * a.chunks;
  const int r = x / a.hkv, g = x - r * a.hkv;
  const int qs = a.cu[r], n = min(a.cu[r + 1], a.total_q) - qs;
  const int L = min(int64_t(a.seq_lens[r]), min(a.w_stride, int64_t(a.max_blocks) * kBlock));
  if (qs < 0 || n <= 0 || a.seq_lens[r] < a.cu[r + 1] - qs) return;
  const int base = a.seq_lens[r] - (a.cu[r + 1] - qs);  // first row's position
  const int G = a.hq / a.hkv, rows = n * G;
  const float c = a.scale_log2;
  const int32_t* bt = a.bt + (int64_t)r * a.max_blocks;

  u32x4 raw[NL];
  float raw_lse = 0.f;
  int raw_pos = 0;
  // the row of unit i, or the row tid for its log-sum-exp
  auto row_of = [&](int rho, int& qi) {
    qi = rho / G;
    return (int64_t)(qs + qi) * a.hq + g * G + (rho - qi * G);
  };
  auto counts = [](float lse) { return fabsf(lse) < __builtin_huge_valf(); };
  auto load_rows = [&](int r0) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = 256 * i + tid, lr = u / UR, p = u % UR;
      raw[i] = zero16();
      if (r0 + lr < rows) {
        int qi;
        const int64_t row = row_of(r0 + lr, qi);
        const u32x4 v = ld16(a.q + row * D + 8 * p);
        if (counts(a.lse[row])) raw[i] = v;
      }
    }
    if (tid < kRows) {
      raw_lse = __builtin_huge_valf();
      raw_pos = -1;
      if (r0 + tid < rows) {
        int qi;
        const float lse = a.lse[row_of(r0 + tid, qi)];
        if (counts(lse)) raw_lse = lse * kLog2e;
        raw_pos = base + qi;
      }
    }
  };
  auto store_rows = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = 256 * i + tid, lr = u / UR, p = u % UR;
      st16(&sm.q[buf][8 * (lr * UR + (p ^ (lr & 7)))], raw[i]);
    }
    if (tid < kRows) sm.lse[buf][tid] = raw_lse, sm.pos[buf][tid] = raw_pos;
  };

  for (int64_t chunk = first_chunk; chunk * kChunk < L; chunk += a.chunks) {
    const int key0 = int(chunk) * kChunk;
    // rows from the first that sees one of the chunk's keys on
    const int row_first = max(0, key0 - base) * G / kRows * kRows;
    load_rows(row_first);
    // the keys: lane (j, hh) holds key j's dims of each k-step
    bf16x8 k[KT][KS];
    int key[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      key[t] = key0 + (w * KT + t) * 32 + j;
      const int kk = min(key[t], L - 1);
      const int64_t b = (int64_t)clamp_block(bt[kk / kBlock], a.num_blocks) * a.hkv + g;
      const int o = kk % kBlock;
      if constexpr (BITS == 16) {
        const __bf16* p = reinterpret_cast<const __bf16*>(a.kc) + b * (kBlock * D) + key_slot_pos(o) * kKeyGroup + 8 * hh;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          k[t][ks] = as_bf16x8(__builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
              p + (ks / 2) * (kBlock * kKeyGroup) + 16 * (ks % 2))));
      } else {
        const uint8_t* p = a.kc + b * (kBlock * D / 2) + o * (D / 2) + hh * (D / 4);
        const uint8_t* s = a.scales + b * ((D / 32 + 1) * kBlock) + hh * (D / 64) * kBlock + o;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 16 * i));
          const float sc = __uint_as_float(uint32_t(s[i * kBlock]) << 23);
#pragma unroll
          for (int u = 0; u < 4; ++u)
            k[t][4 * i + u] = as_bf16x8(u32x4{
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[u], sc, 0)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[u], sc, 1)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[u], sc, 2)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[u], sc, 3))});
        }
      }
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
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        // the dims of k-step ks: as the keys' lanes hold them
        const int p = BITS == 16 ? 2 * ks + hh : hh * KS + ks;
        const bf16x8 q = as_bf16x8(ld16(&sm.q[buf][8 * (j * UR + (p ^ (j & 7)))]));
#pragma unroll
        for (int t = 0; t < KT; ++t) s[t] = mfma32(q, k[t][ks], s[t]);
      }
      const bool masked = base + r0 / G < last_key;  // the first row does not see all keys
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        if (r0 + 8 * q4 >= rows) break;
        const f32x4 z = *reinterpret_cast<const f32x4*>(&sm.lse[buf][8 * q4 + 4 * hh]);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float p = fast_exp2(fmaf(s[t][4 * q4 + e], c, -z[e]));
            if (masked) p = key[t] <= sm.pos[buf][8 * q4 + 4 * hh + e] ? p : 0.f;
            sum[t] += p;
          }
      }
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

}  // namespace

int launch_attn_weights(const void* q, const float* lse, const void* kc, const uint8_t* scales,
                        int32_t num_blocks, const int32_t* bt, int32_t max_blocks,
                        const int32_t* seq_lens, const int32_t* cu, int32_t n_seqs, int32_t total_q,
                        int32_t hq, int32_t hkv, int32_t d, int32_t bits, float scale, float* w,
                        int64_t w_stride, bool add, hipStream_t stream) {
  WeightArgs a{static_cast<const __bf16*>(q), lse, static_cast<const uint8_t*>(kc), scales, bt, seq_lens,
               cu, w, w_stride, max_blocks, num_blocks, total_q, hq, hkv, 0, scale * kLog2e, add};
  const int64_t heads = int64_t(n_seqs) * hkv, keys = min(w_stride, int64_t(max_blocks) * kBlock);
  const bool wide = int64_t(total_q) * (hq / hkv) > 32 * int64_t(n_seqs);
  const int64_t chunk = wide ? 256 : 128;
  int64_t chunks = (keys + chunk - 1) / chunk;
  // few workgroups without keys where the array is wider than the sequences are long
  chunks = min(chunks, max(int64_t(1), 32768 / heads));
  if (heads * chunks > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
  a.chunks = int32_t(chunks);
  const dim3 grid(unsigned(heads * chunks));
#define PA_W(DD, BB, KK) hipLaunchKernelGGL((attn_weights_kernel<DD, BB, KK>), grid, dim3(256), 0, stream, a)
#define PA_W_BITS(DD)                 \
  if (bits == 16) {                   \
    if (wide) PA_W(DD, 16, 2);        \
    else PA_W(DD, 16, 1);             \
  } else {                            \
    if (wide) PA_W(DD, 4, 2);         \
    else PA_W(DD, 4, 1);              \
  }
  if (d == 128) {
    PA_W_BITS(128)
  } else {
    PA_W_BITS(64)
  }
#undef PA_W_BITS
#undef PA_W
  return static_cast<int>(hipGetLastError());
}

}  // namespace dev
}  // namespace pa
