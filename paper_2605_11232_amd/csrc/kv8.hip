// The 8-bit cache: append (quantise) and read back.
//
// A (block, kv-head) holds 16 tokens of e4m3 keys [D/64][16][64] and values
// [D][16], and a power-of-two scale for each of the two (a byte, exponent + 127).
// One workgroup owns one (sequence, block, kv-head) of the launch, so that the
// scale, which needs all of the block's new tokens, and the codes of earlier
// tokens, which are rounded again where the scale grows, are found and written by
// one workgroup: no atomics and no second launch, and the result does not depend
// on how the work is split.
//
// Workgroups find their block in cu_seqlens: sequence r owns the slots
// cu[r] / 16 + 2 r up to the next sequence's first, at least as many as the
// blocks that its rows touch (n rows touch at most n / 16 + 2).
#include "device_common.h"

namespace pa {
namespace dev {
namespace {

constexpr int kExpMin = -100, kExpMax = 120, kExpBias = 127;

struct Kv8Args {
  const int32_t* bt;
  const int32_t* seq_lens;
  const int32_t* cu;
  uint8_t* kc;
  uint8_t* vc;
  uint8_t* scales;
  int64_t k_stride, v_stride;
  int32_t max_blocks, n_seqs, n_tokens, num_blocks, hkv;
};

// One block of the launch and its rows.
struct BlockRows {
  int64_t bh;      // block * hkv + kv-head; -1: nothing to do
  int off0, off1;  // token offsets [off0, off1) of the block have rows
  int row0;        // row of offset off0
};

// Largest r of [0, n) with cu[r] / 16 + 2 r <= x: each round compares 64 evenly
// spaced sequences, one per lane.
__device__ __forceinline__ int find_seq(const int32_t* cu, int n, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + lane * step;
    const bool below = i < hi && cu[i < hi ? i : lo] / kBlock + 2 * i <= x;
    const int c = max(1, __popcll(__ballot(below)));
    lo += (c - 1) * step;
    hi = min(lo + step, hi);
  }
  return lo;
}

__device__ __forceinline__ BlockRows find_rows(const Kv8Args& a, int slot, int h) {
  BlockRows b{-1, 0, 0, 0};
  const int r = find_seq(a.cu, a.n_seqs, slot);
  const int c0 = a.cu[r], n = a.cu[r + 1] - c0, L = a.seq_lens[r];
  const int first = L - n;  // first row's position
  if (n <= 0 || first < 0 || c0 < 0) return b;
  const int64_t j = first / kBlock + (int64_t)slot - (c0 / kBlock + 2 * r);
  if (j < 0 || j * kBlock >= L || j >= a.max_blocks) return b;
  const int p0 = int(j) * kBlock;
  b.off0 = max(first - p0, 0);
  b.off1 = min(L - p0, kBlock);
  b.row0 = c0 + p0 + b.off0 - first;
  const int id = a.bt[(int64_t)r * a.max_blocks + j];
  // rows past the caller's: cu does not end at n_tokens
  if (id >= 0 && id < a.num_blocks && (int64_t)b.row0 + (b.off1 - b.off0) <= a.n_tokens)
    b.bh = (int64_t)id * a.hkv + h;
  return b;
}

// Smallest e of [kExpMin, kExpMax] with amax <= 448 * 2^e; 448 = 1.75 * 2^8.
__device__ __forceinline__ int exponent_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = int(u >> 23) - 127 - 8 + ((u & 0x7FFFFF) > 0x600000 ? 1 : 0);
  return min(max(e, kExpMin), kExpMax);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }

typedef float f32x2 __attribute__((ext_vector_type(2)));

// x0 * s, x1 * s, ... as e4m3 codes (nearest even; all at most 448, or NaN).
__device__ __forceinline__ uint32_t codes_of(float x0, float x1, float x2, float x3, float s) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(x0 * s, x1 * s, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(x2 * s, x3 * s, r, true));
}
// Codes rounded again for a scale 1 / s times as large.
__device__ __forceinline__ uint32_t codes_again(uint32_t c, float s) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  return codes_of(a[0], a[1], b[0], b[1], s);
}
// The first `keep` (any int) bytes of old, the rest of x.
__device__ __forceinline__ uint32_t first_bytes(uint32_t old, uint32_t x, int keep) {
  const int k = min(max(keep, 0), 4);
  const uint32_t m = k == 4 ? ~0u : (1u << (8 * k)) - 1u;
  return (old & m) | (x & ~m);
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
template <>
__device__ __forceinline__ void load8<__bf16>(const __bf16* p, float (&x)[8]) {
  const bf16x8 a = as_bf16x8(ld16(p));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = float(a[i]);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_append_kernel(const T* __restrict__ k_new,
                                                         const T* __restrict__ v_new, Kv8Args a) {
  constexpr int CH = D / 8;             // 8-dim chunks of a row
  constexpr int U = 2 * kBlock * CH / 256;  // chunks of K and V per thread
  __shared__ float amax_sh[2][4];
  __shared__ uint8_t vt[kBlock][D + 8];
  const int tid = threadIdx.x, w = tid >> 6;
  const int h = blockIdx.x % a.hkv;
  const BlockRows b = find_rows(a, blockIdx.x / a.hkv, h);
  if (b.bh < 0) return;

  // chunk c of thread tid: K's for c < 16 CH, V's after; token offset, then dims
  float x[U][8];
  float mx[2] = {0.f, 0.f};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = u * 256 + tid, side = c / (kBlock * CH);
    const int o = c / CH % kBlock, part = c % CH;
    if (o < b.off0 || o >= b.off1) continue;
    const int64_t row = b.row0 + o - b.off0;
    load8((side ? v_new + row * a.v_stride : k_new + row * a.k_stride) + (int64_t)h * D + 8 * part, x[u]);
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool finite = fabsf(x[u][i]) < __builtin_huge_valf();
      m = fmaxf(m, finite ? fabsf(x[u][i]) : 0.f);
      x[u][i] = finite ? x[u][i] : __builtin_nanf("");
    }
    if (side) mx[1] = fmaxf(mx[1], m);
    else mx[0] = fmaxf(mx[0], m);
  }
#pragma unroll
  for (int s = 0; s < 2; ++s) {
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) mx[s] = fmaxf(mx[s], wave_xor(mx[s], k));
    if ((tid & 63) == 0) amax_sh[s][w] = mx[s];
  }
  __syncthreads();
  int e[2], grow[2];  // exponents, and how far they grew for earlier tokens
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    e[s] = exponent_of(fmaxf(fmaxf(amax_sh[s][0], amax_sh[s][1]), fmaxf(amax_sh[s][2], amax_sh[s][3])));
    grow[s] = 0;
    if (b.off0 > 0) {
      // (bounded: the earlier tokens may never have been stored)
      const int was = min(max(int(a.scales[2 * b.bh + s]) - kExpBias, kExpMin), kExpMax);
      grow[s] = min(max(e[s] - was, 0), 126);
      e[s] = max(e[s], was);
    }
  }
  __syncthreads();  // every thread has read the scales
  if (tid < 2) a.scales[2 * b.bh + tid] = uint8_t((tid ? e[1] : e[0]) + kExpBias);

  uint8_t* kb = a.kc + b.bh * (kBlock * D);
  uint8_t* vb = a.vc + b.bh * (kBlock * D);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = u * 256 + tid, side = c / (kBlock * CH);
    const int o = c / CH % kBlock, part = c % CH;
    if (o < b.off0 || o >= b.off1) continue;
    const float s = pow2(-(side ? e[1] : e[0]));
    const u32x2 q = {codes_of(x[u][0], x[u][1], x[u][2], x[u][3], s),
                     codes_of(x[u][4], x[u][5], x[u][6], x[u][7], s)};
    if (side) *reinterpret_cast<u32x2*>(&vt[o][8 * part]) = q;
    else *reinterpret_cast<u32x2*>(kb + part / 8 * 1024 + o * 64 + part % 8 * 8) = q;
  }
  if (grow[0] > 0) {  // earlier tokens' keys
    const float s = pow2(-grow[0]);
    for (int c = tid; c < b.off0 * (D / 16); c += 256) {
      uint8_t* p = kb + c % (D / 64) * 1024 + c / (D / 16) * 64 + c / (D / 64) % 4 * 16;
      u32x4 v = ld16(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = codes_again(v[i], s);
      st16(p, v);
    }
  }
  __syncthreads();
  const bool whole = b.off0 == 0 && b.off1 == kBlock;
  if (whole || grow[1] > 0) {
    const float s = pow2(-grow[1]);
    for (int d = tid; d < D; d += 256) {
      u32x4 v = zero16();
      if (!whole) v = ld16(vb + d * kBlock);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t q = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) q |= uint32_t(vt[4 * i + k][d]) << (8 * k);
        // earlier tokens, new ones, and slots behind them as they were
        if (!whole)
          q = first_bytes(codes_again(v[i], s), first_bytes(q, v[i], b.off1 - 4 * i), b.off0 - 4 * i);
        v[i] = q;
      }
      st16(vb + d * kBlock, v);
    }
  } else {
    for (int c = tid; c < D * (b.off1 - b.off0); c += 256) {
      const int d = c % D, o = b.off0 + c / D;
      vb[d * kBlock + o] = vt[o][d];
    }
  }
}

// Eight e4m3 codes times a power of two, stored as T.
template <typename T>
__device__ __forceinline__ void store8(T* p, u32x2 c, float s);
template <>
__device__ __forceinline__ void store8<float>(float* p, u32x2 c, float s) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c[i], false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(c[i], true);
    *reinterpret_cast<f32x4*>(p + 4 * i) = f32x4{a[0] * s, a[1] * s, b[0] * s, b[1] * s};
  }
}
template <>
__device__ __forceinline__ void store8<__bf16>(__bf16* p, u32x2 c, float s) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], s, false));
    r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], s, true));
  }
  st16(p, r);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_read_kernel(T* __restrict__ k_out, T* __restrict__ v_out,
                                                       Kv8Args a) {
  constexpr int CH = D / 8;
  __shared__ uint8_t vt[kBlock][D + 8];
  const int tid = threadIdx.x;
  const int h = blockIdx.x % a.hkv;
  const BlockRows b = find_rows(a, blockIdx.x / a.hkv, h);
  if (b.bh < 0) return;
  const uint8_t* kb = a.kc + b.bh * (kBlock * D);
  const uint8_t* vb = a.vc + b.bh * (kBlock * D);
  const float sk = pow2(int(a.scales[2 * b.bh]) - kExpBias);
  const float sv = pow2(int(a.scales[2 * b.bh + 1]) - kExpBias);
  for (int d = tid; d < D; d += 256) {
    const u32x4 v = ld16(vb + d * kBlock);
#pragma unroll
    for (int o = 0; o < kBlock; ++o) vt[o][d] = uint8_t(v[o / 4] >> (8 * (o % 4)));
  }
  for (int c = tid; c < kBlock * CH; c += 256) {
    const int o = c / CH, part = c % CH;
    if (o < b.off0 || o >= b.off1) continue;
    const u32x2 q = *reinterpret_cast<const u32x2*>(kb + part / 8 * 1024 + o * 64 + part % 8 * 8);
    store8(k_out + (int64_t)(b.row0 + o - b.off0) * a.k_stride + (int64_t)h * D + 8 * part, q, sk);
  }
  __syncthreads();
  for (int c = tid; c < kBlock * CH; c += 256) {
    const int o = c / CH, part = c % CH;
    if (o < b.off0 || o >= b.off1) continue;
    const u32x2 q = *reinterpret_cast<const u32x2*>(&vt[o][8 * part]);
    store8(v_out + (int64_t)(b.row0 + o - b.off0) * a.v_stride + (int64_t)h * D + 8 * part, q, sv);
  }
}

// Workgroups of n rows of n_seqs sequences.
int64_t kv8_grid(int32_t n, int32_t n_seqs, int32_t hkv) {
  return (int64_t(n) / kBlock + 2 * int64_t(n_seqs)) * hkv;
}

}  // namespace

int launch_kv8_append(const void* kn, int64_t k_stride, const void* vn, int64_t v_stride,
                      const int32_t* bt, int32_t max_blocks, const int32_t* seq_lens,
                      const int32_t* cu, int32_t n_seqs, int32_t n, void* kc, void* vc,
                      uint8_t* scales, int32_t nb, int32_t hkv, int32_t d, int32_t dtype,
                      hipStream_t stream) {
  const Kv8Args a{bt, seq_lens, cu, static_cast<uint8_t*>(kc), static_cast<uint8_t*>(vc), scales,
                  k_stride, v_stride, max_blocks, n_seqs, n, nb, hkv};
  const int64_t grid = kv8_grid(n, n_seqs, hkv);
  if (grid > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
#define PA_KV8(T, DD)                                                                            \
  hipLaunchKernelGGL((kv8_append_kernel<T, DD>), dim3(unsigned(grid)), dim3(256), 0, stream,     \
                     static_cast<const T*>(kn), static_cast<const T*>(vn), a)
  if (dtype == 1) {
    if (d == 128) PA_KV8(__bf16, 128);
    else PA_KV8(__bf16, 64);
  } else {
    if (d == 128) PA_KV8(float, 128);
    else PA_KV8(float, 64);
  }
#undef PA_KV8
  return static_cast<int>(hipGetLastError());
}

int launch_kv8_read(void* k_out, int64_t k_stride, void* v_out, int64_t v_stride,
                    const int32_t* bt, int32_t max_blocks, const int32_t* seq_lens,
                    const int32_t* cu, int32_t n_seqs, int32_t n, const void* kc, const void* vc,
                    const uint8_t* scales, int32_t nb, int32_t hkv, int32_t d, int32_t dtype,
                    hipStream_t stream) {
  const Kv8Args a{bt, seq_lens, cu, static_cast<uint8_t*>(const_cast<void*>(kc)),
                  static_cast<uint8_t*>(const_cast<void*>(vc)), const_cast<uint8_t*>(scales),
                  k_stride, v_stride, max_blocks, n_seqs, n, nb, hkv};
  const int64_t grid = kv8_grid(n, n_seqs, hkv);
  if (grid > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
#define PA_KV8(T, DD)                                                                            \
  hipLaunchKernelGGL((kv8_read_kernel<T, DD>), dim3(unsigned(grid)), dim3(256), 0, stream,       \
                     static_cast<T*>(k_out), static_cast<T*>(v_out), a)
  if (dtype == 1) {
    if (d == 128) PA_KV8(__bf16, 128);
    else PA_KV8(__bf16, 64);
  } else {
    if (d == 128) PA_KV8(float, 128);
    else PA_KV8(float, 64);
  }
#undef PA_KV8
  return static_cast<int>(hipGetLastError());
}

}  // namespace dev
}  // namespace pa
