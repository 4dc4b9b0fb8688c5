// The 4-bit cache: append (quantise) and read back.
//
// A (block, kv-head) holds 16 tokens of e2m1 codes, two in a byte (the first in the low
// half): keys [16][D/2], a token's dims side by side; values [D/32][16][2][8], dim 32 c +
// 16 a + i at [c][i][a], a byte of it two neighbouring tokens, so that attention takes 16
// keys of dims d and d + 16 in one 16-byte load.  Scales [D/32 + 1][16] are bytes: for
// each token, a power of two for 32 dims of its key (rows 0 .. D/32 - 1) and one for its
// value (the last row).
//
// As in the 8-bit cache one wavefront owns one (sequence, block, kv-head) of the launch:
// two tokens' value codes share a byte, which one wavefront reads, changes and writes.
// Scales belong to one token, so earlier tokens' codes stay as they are.
#include <type_traits>

#include "kv_rows.h"

namespace pa {
namespace dev {
namespace {

constexpr int kExpMin = -100, kExpMax = 100;
constexpr uint32_t kScaleNan = 255;  // a part with a value that is not finite

// Smallest e of [kExpMin, kExpMax] with amax <= 7 * 2^e; 7 = 1.75 * 2^2.
__device__ __forceinline__ int exponent_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = int(u >> 23) - 127 - 2 + ((u & 0x7FFFFF) > 0x600000 ? 1 : 0);
  return min(max(e, kExpMin), kExpMax);
}

// Codes of eight values / s (a power of two): nearest even, 6 where that is more.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], float s) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
}

// Transpose of 8 x 8 codes: code i of word k becomes code k of word i.
__device__ __forceinline__ void transpose8(uint32_t (&w)[8]) {
  constexpr uint32_t kLow = 0x0F0F0F0F;
  uint32_t lo[4], hi[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    lo[m] = (w[2 * m] & kLow) | (w[2 * m + 1] & kLow) << 4;
    hi[m] = (w[2 * m] >> 4 & kLow) | (w[2 * m + 1] & ~kLow);
  }
  transpose4(lo);
  transpose4(hi);
#pragma unroll
  for (int m = 0; m < 4; ++m) w[2 * m] = lo[m], w[2 * m + 1] = hi[m];
}

// Word of (dim d, token half h) in a block's values: 8 tokens.
__device__ __forceinline__ int value_word(int d, int h) {
  return (d / 32) * 64 + (d % 16) * 4 + (d / 16 % 2) * 2 + h;
}

// One wavefront per (block, kv-head).  D / 8 lanes hold a token's keys, the next as many
// its values, 8 dims a lane; 64 / (D / 4) tokens at a time, all loads issued before the
// first is used.  The keys' codes go straight to the cache, the values' through LDS, where
// D / 4 lanes take a square of 8 dims x 8 tokens each and transpose it; then each lane
// stores 16 bytes, codes of tokens without rows as they were.  Bound by the rows' bytes where
// there are many (64 prompts of 256-1024 tokens, 8 kv-heads of 128: 173 MB read, 45 written,
// 49 us, 4.5 TB/s), by latency where there are few (a token of 256 sequences 4.8 us).
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(const T* __restrict__ k_new,
                                                         const T* __restrict__ v_new, KvRowArgs a) {
  constexpr int LR = D / 8;            // lanes of a row
  constexpr int TI = 64 / (2 * LR);    // tokens at a time
  constexpr int NI = kBlock / TI;
  constexpr int NS = D / 32 + 1;       // scale rows
  __shared__ __align__(16) uint32_t vt_sh[4][kBlock][LR + 1];
  __shared__ __align__(16) uint32_t vb_sh[4][2 * D];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i = (int64_t)blockIdx.x * 4 + w;
  const int64_t slot = i / a.hkv;
  if (slot >= a.slots) return;
  const int h = int(i - slot * a.hkv);
  const BlockRows b = find_rows(a, int(slot));
  if (b.off0 == b.off1) return;
  uint32_t (*vt)[LR + 1] = vt_sh[w];
  uint32_t* vn = vb_sh[w];
  const int c = lane % LR, side = lane / LR % 2, sub = lane / (2 * LR);
  Raw8<T> x[NI];
  const T* src = (side ? v_new + (int64_t)b.row0 * a.v_stride : k_new + (int64_t)b.row0 * a.k_stride) + (int64_t)h * D + 8 * c;
  const int64_t stride = side ? a.v_stride : a.k_stride;
  auto has = [&](int u) { return u * TI + sub >= b.off0 && u * TI + sub < b.off1; };
#pragma unroll
  for (int u = 0; u < NI; ++u)
    if (has(u)) x[u].load(src + (u * TI + sub - b.off0) * stride);
  // the rows are on their way while the block's id arrives
  if (b.id < 0 || b.id >= a.num_blocks) return;
  const int64_t bh = (int64_t)b.id * a.hkv + h;
  uint8_t* kb = a.kc + bh * (kBlock * D / 2);
  u32x4* vb = reinterpret_cast<u32x4*>(a.vc + bh * (kBlock * D / 2)) + lane;
  uint8_t* sb = a.scales + bh * (NS * kBlock);
  const bool whole = b.off0 == 0 && b.off1 == kBlock;
  u32x4 was = zero16();
  if (!whole && lane < D / 2) was = *vb;
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    if (!has(u)) continue;  // lanes of one part agree
    float y[8], mx = 0.f;
    bool ok = true;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      y[k] = x[u].at(k);
      ok = ok && fabsf(y[k]) < __builtin_huge_valf();
      mx = fmaxf(mx, fabsf(y[k]));
    }
    if (!ok) mx = __builtin_huge_valf();
    // a key's scale is 32 dims', of 4 lanes; a value's the row's
    mx = fmaxf(mx, wave_xor(mx, 1));
    mx = fmaxf(mx, wave_xor(mx, 2));
#pragma unroll
    for (int m = 4; m < LR; m <<= 1) {
      const float other = wave_xor(mx, m);
      if (side) mx = fmaxf(mx, other);
    }
    ok = mx < __builtin_huge_valf();
    const int e = exponent_of(mx), o = u * TI + sub;
    const uint32_t q = ok ? codes_of(y, pow2(e)) : 0;
    const uint8_t byte = uint8_t(ok ? uint32_t(e + kExpBias) : kScaleNan);
    if (side) {
      vt[o][c] = q;
      if (c == 0) sb[(NS - 1) * kBlock + o] = byte;
    } else {
      *reinterpret_cast<uint32_t*>(kb + o * (D / 2) + 4 * c) = q;
      if (c % 4 == 0) sb[c / 4 * kBlock + o] = byte;
    }
  }
  wave_lds_order();
  if (lane < D / 4) {
    const int dw = lane % LR, half = lane / LR;
    uint32_t q[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) q[k] = vt[8 * half + k][dw];
    transpose8(q);
#pragma unroll
    for (int k = 0; k < 8; ++k) vn[value_word(8 * dw + k, half)] = q[k];
  }
  wave_lds_order();
  if (lane < D / 2) {
    u32x4 v = ld16(vn + 4 * lane);
    if (!whole) {
      // codes [off0, off1) of a dim's 16
      const uint64_t m = (b.off1 == kBlock ? ~0ull : (1ull << (4 * b.off1)) - 1) & ~((1ull << (4 * b.off0)) - 1);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t mk = uint32_t(m >> (32 * (k % 2)));
        v[k] = (v[k] & mk) | (was[k] & ~mk);
      }
    }
    *vb = v;
  }
}

// Codes times a power of two (or NaN), 16 bytes of them stored as T: eight bf16 numbers, or
// the four low codes in float32.
template <typename T>
__device__ __forceinline__ void store16(T* p, uint32_t c, float s) {
  if constexpr (sizeof(T) == 2) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
    __builtin_nontemporal_store(s == s ? r : u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u},
                                reinterpret_cast<u32x4*>(p));
  } else {
    const f32x2 r0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 0), r1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 1);
    __builtin_nontemporal_store(f32x4{r0[0] * s, r0[1] * s, r1[0] * s, r1[1] * s}, reinterpret_cast<f32x4*>(p));
  }
}

// Power of two of a scale byte, NaN for 255.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return byte == kScaleNan ? __builtin_nanf("") : __uint_as_float(byte << 23);
}

// One wavefront per (block, kv-head), all loads issued before the first store.  16 bytes of a
// token's row a lane, so that a store is of whole lines (float32 rows written as two halves of
// 32 bytes a lane took 191 us for 64 x 640 tokens, 63 this way); the values' codes are
// transposed on the way, as in append.  Bound by what it writes, past the caches: 16 sequences
// of 4096-12000 tokens, 8 kv-heads of 128, 524 MB written, 138 read, 119 us, 5.6 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(T* __restrict__ k_out, T* __restrict__ v_out,
                                                       KvRowArgs a) {
  constexpr int W = D / 8;           // words of a token's codes
  constexpr int PD = 16 / sizeof(T); // dims of a lane
  constexpr int LR = D / PD;         // lanes of a token
  constexpr int TI = 64 / LR;        // tokens at a time
  typedef typename std::conditional<PD == 8, uint32_t, uint16_t>::type Codes;
  constexpr int NI = kBlock / TI;
  constexpr int NS = D / 32 + 1;
  __shared__ __align__(16) uint32_t vt_sh[4][kBlock][W + 1];
  __shared__ __align__(16) uint32_t vb_sh[4][2 * D];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i = (int64_t)blockIdx.x * 4 + w;
  const int64_t slot = i / a.hkv;
  if (slot >= a.slots) return;
  const int h = int(i - slot * a.hkv);
  const BlockRows b = find_rows(a, int(slot));
  if (b.off0 == b.off1 || b.id < 0 || b.id >= a.num_blocks) return;
  const int64_t bh = (int64_t)b.id * a.hkv + h;
  const Codes* kb = reinterpret_cast<const Codes*>(a.kc + bh * (kBlock * D / 2));
  const uint8_t* vb = a.vc + bh * (kBlock * D / 2);
  const uint8_t* sb = a.scales + bh * (NS * kBlock);
  uint32_t (*vt)[W + 1] = vt_sh[w];
  uint32_t* vn = vb_sh[w];
  const int c = lane % LR, sub = lane / LR;
  Codes k[NI];
  uint8_t sk[NI], sv[NI];
  u32x4 v = zero16();
  if (lane < D / 2) v = ld16(vb + 16 * lane);
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    k[u] = kb[u * 64 + lane];
    sk[u] = sb[c * PD / 32 * kBlock + u * TI + sub];
    sv[u] = sb[(NS - 1) * kBlock + u * TI + sub];
  }
  if (lane < D / 2) st16(vn + 4 * lane, v);
  wave_lds_order();
  if (lane < D / 4) {
    const int dw = lane % W, half = lane / W;
    uint32_t q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = vn[value_word(8 * dw + j, half)];
    transpose8(q);
#pragma unroll
    for (int j = 0; j < 8; ++j) vt[8 * half + j][dw] = q[j];
  }
  wave_lds_order();
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    const int o = u * TI + sub;
    if (o < b.off0 || o >= b.off1) continue;
    const int64_t row = b.row0 + o - b.off0;
    const uint32_t v_codes = PD == 8 ? vt[o][c] : vt[o][c / 2] >> (16 * (c % 2));
    store16(k_out + row * a.k_stride + (int64_t)h * D + PD * c, k[u], scale_of(sk[u]));
    store16(v_out + row * a.v_stride + (int64_t)h * D + PD * c, v_codes, scale_of(sv[u]));
  }
}

}  // namespace

int launch_kv4_append(const void* kn, int64_t k_stride, const void* vn, int64_t v_stride,
                      const int32_t* bt, int32_t max_blocks, const int32_t* seq_lens,
                      const int32_t* cu, int32_t n_seqs, int32_t n, void* kc, void* vc,
                      uint8_t* scales, int32_t nb, int32_t hkv, int32_t d, int32_t dtype,
                      hipStream_t stream) {
  const KvRowArgs a = with_slots({bt, seq_lens, cu, static_cast<uint8_t*>(kc), static_cast<uint8_t*>(vc), scales,
                  k_stride, v_stride, max_blocks, n_seqs, n, nb, hkv, 0, false});
  const int64_t grid = (a.slots * hkv + 3) / 4;  // a wavefront per (block, kv-head)
  if (grid > INT32_MAX || a.slots > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
#define PA_KV4(T, DD)                                                                            \
  hipLaunchKernelGGL((kv4_append_kernel<T, DD>), dim3(unsigned(grid)), dim3(256), 0, stream,     \
                     static_cast<const T*>(kn), static_cast<const T*>(vn), a)
  if (dtype == 1) {
    if (d == 128) PA_KV4(__bf16, 128);
    else PA_KV4(__bf16, 64);
  } else {
    if (d == 128) PA_KV4(float, 128);
    else PA_KV4(float, 64);
  }
#undef PA_KV4
  return static_cast<int>(hipGetLastError());
}

int launch_kv4_read(void* k_out, int64_t k_stride, void* v_out, int64_t v_stride,
                    const int32_t* bt, int32_t max_blocks, const int32_t* seq_lens,
                    const int32_t* cu, int32_t n_seqs, int32_t n, const void* kc, const void* vc,
                    const uint8_t* scales, int32_t nb, int32_t hkv, int32_t d, int32_t dtype,
                    hipStream_t stream) {
  const KvRowArgs a = with_slots({bt, seq_lens, cu, static_cast<uint8_t*>(const_cast<void*>(kc)),
                  static_cast<uint8_t*>(const_cast<void*>(vc)), const_cast<uint8_t*>(scales),
                  k_stride, v_stride, max_blocks, n_seqs, n, nb, hkv, 0, false});
  const int64_t grid = (a.slots * hkv + 3) / 4;
  if (grid > INT32_MAX || a.slots > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
#define PA_KV4(T, DD)                                                                            \
  hipLaunchKernelGGL((kv4_read_kernel<T, DD>), dim3(unsigned(grid)), dim3(256), 0, stream,       \
                     static_cast<T*>(k_out), static_cast<T*>(v_out), a)
  if (dtype == 1) {
    if (d == 128) PA_KV4(__bf16, 128);
    else PA_KV4(__bf16, 64);
  } else {
    if (d == 128) PA_KV4(float, 128);
    else PA_KV4(float, 64);
  }
#undef PA_KV4
  return static_cast<int>(hipGetLastError());
}

}  // namespace dev
}  // namespace pa
