// The 8-bit cache: append (quantise) and read back.
//
// A (block, kv-head) holds 16 tokens of e4m3 keys [D/64][16][64] and values
// [D][16], and a power-of-two scale for each of the two (a byte, exponent + 127).
// One wavefront owns one (sequence, block, kv-head) of the
// launch, so that the scale, which needs all of the block's new tokens, and the codes
// of earlier tokens, which are rounded again where the scale grows, are found and
// written by one: no atomics and no second launch, and the result does not depend on
// how the work is split.
//
// They find their block in cu_seqlens: sequence r owns the slots cu[r] / 16 + 2 r up
// to the next sequence's first, at least as many as the blocks that its rows touch (n
// rows touch at most n / 16 + 2); or each row a slot, of which a block's first one
// does the work.
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

__device__ __forceinline__ BlockRows find_rows(const Kv8Args& a, int slot) {
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
// Codes of the largest scale: finite values from 248 * 2^120 on were rounded to 256, which
// would stand for 2^128; the code below does instead.  Byte by byte, without carries.
__device__ __forceinline__ uint32_t below_256(uint32_t c) {
  const uint32_t other = ((c & 0x7F7F7F7F) ^ 0x78787878) + 0x7F7F7F7F;  // bit 7: not +-256
  return c - ((~other & 0x80808080) >> 7);
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

// Eight values of T as loaded, and as float32.  Non-temporal: the rows are read once (64
// prompts whose rows are in no cache 49 us, 55 with plain loads; 46 where the last-level
// cache holds them all).
template <typename T>
struct Raw8 {
  u32x4 x[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (size_t i = 0; i < sizeof(T) / 2; ++i) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 16 / sizeof(T) * i));
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 2) return __uint_as_float(i % 2 ? x[0][i / 2] & 0xFFFF0000u : x[0][i / 2] << 16);
    else return __uint_as_float(x[i / 4][i % 4]);
  }
};

// Order of a wavefront's own LDS accesses: the hardware keeps it, this the compiler.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Transpose of 4 x 4 bytes: byte i of word k becomes byte k of word i.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
  w[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
  w[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
  w[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

// One wavefront per (block, kv-head).  D / 8 lanes hold a token's keys, the next as
// many its values, 8 dims a lane; 64 / (D / 4) tokens at a time, all loads issued
// before the first is used.  The keys' codes go straight to the cache, the values'
// through LDS, where a lane takes a square of 4 dims x 4 tokens and transposes it.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_append_kernel(const T* __restrict__ k_new,
                                                         const T* __restrict__ v_new, Kv8Args a) {
  constexpr int LR = D / 8;            // lanes of a row
  constexpr int TI = 64 / (2 * LR);    // tokens at a time
  constexpr int NI = kBlock / TI;
  constexpr int SQ = D / 64;           // squares of a lane
  __shared__ __align__(16) uint8_t vt_sh[4][kBlock][D + 8];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i = (int64_t)blockIdx.x * 4 + w;
  const int64_t slot = i / a.hkv;
  if (slot >= a.slots) return;
  const int h = int(i - slot * a.hkv);
  const BlockRows b = find_rows(a, int(slot));
  if (b.off0 == b.off1) return;
  uint8_t (*vt)[D + 8] = vt_sh[w];
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
  const int e_old = min(max(int(a.scales[2 * bh + side]) - kExpBias, kExpMin), kExpMax);
  float mx = 0.f;
#pragma unroll
  for (int u = 0; u < NI; ++u)
    if (has(u))
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float v = fabsf(x[u].at(k));
        mx = fmaxf(mx, v < __builtin_huge_valf() ? v : 0.f);
      }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1)
    if (m != LR) mx = fmaxf(mx, wave_xor(mx, m));
  int e = exponent_of(mx), grow = 0;  // of this lane's side; how far it grew for earlier tokens
  if (b.off0 > 0) {
    grow = min(max(e - e_old, 0), 126);
    e = max(e, e_old);
  }
  if (sub == 0 && c == 0) a.scales[2 * bh + side] = uint8_t(e + kExpBias);

  uint8_t* kb = a.kc + bh * (kBlock * D);
  uint8_t* vb = a.vc + bh * (kBlock * D);
  const float s = pow2(-e);
#pragma unroll
  for (int u = 0; u < NI; ++u)
    if (has(u)) {
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float v = x[u].at(k);
        y[k] = fabsf(v) < __builtin_huge_valf() ? v : __builtin_nanf("");
      }
      u32x2 q = {codes_of(y[0], y[1], y[2], y[3], s), codes_of(y[4], y[5], y[6], y[7], s)};
      if (e == kExpMax) q = u32x2{below_256(q[0]), below_256(q[1])};
      const int o = u * TI + sub;
      *reinterpret_cast<u32x2*>(side ? &vt[o][8 * c] : kb + c / 8 * 1024 + o * 64 + c % 8 * 8) = q;
    }
  const int grow_k = __builtin_amdgcn_readlane(grow, 0), grow_v = __builtin_amdgcn_readlane(grow, LR);
  if (grow_k > 0) {  // earlier tokens' keys
    const float f = pow2(-grow_k);
    for (int j = lane; j < b.off0 * (D / 16); j += 64) {
      uint8_t* p = kb + j % (D / 64) * 1024 + j / (D / 16) * 64 + j / (D / 64) % 4 * 16;
      u32x4 v = ld16(p);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = codes_again(v[k], f);
      st16(p, v);
    }
  }
  wave_lds_order();
  const bool whole = b.off0 == 0 && b.off1 == kBlock;
  if (whole || grow_v > 0) {
    const float f = pow2(-grow_v);
    const int dq = 4 * (lane % (D / 4)), o0 = 4 * SQ * (lane / (D / 4));
    uint32_t q[SQ][4];
#pragma unroll
    for (int sq = 0; sq < SQ; ++sq) {
#pragma unroll
      for (int k = 0; k < 4; ++k) q[sq][k] = *reinterpret_cast<const uint32_t*>(&vt[o0 + 4 * sq + k][dq]);
      transpose4(q[sq]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t* p = reinterpret_cast<uint32_t*>(vb + (dq + k) * kBlock + o0);
      uint32_t r[SQ];
#pragma unroll
      for (int sq = 0; sq < SQ; ++sq) {
        r[sq] = q[sq][k];
        if (!whole) {
          // earlier tokens, new ones, and slots behind them as they were
          const uint32_t was = p[sq];
          const int o = o0 + 4 * sq;
          r[sq] = first_bytes(codes_again(was, f), first_bytes(r[sq], was, b.off1 - o), b.off0 - o);
        }
      }
      if constexpr (SQ == 2) *reinterpret_cast<u32x2*>(p) = u32x2{r[0], r[1]};
      else p[0] = r[0];
    }
  } else {
    for (int j = lane; j < D * (b.off1 - b.off0); j += 64) {
      const int d = j % D, o = b.off0 + j / D;
      vb[d * kBlock + o] = vt[o][d];
    }
  }
}

// Four e4m3 codes times a power of two, stored as T.  Non-temporal: the rows leave the
// caches to what is read again (163000 tokens 146 us, 156 with plain stores).
template <typename T>
__device__ __forceinline__ void store4(T* p, uint32_t c, float s) {
  if constexpr (sizeof(T) == 2) {
    __builtin_nontemporal_store(u32x2{
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, false)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, true))}, reinterpret_cast<u32x2*>(p));
  } else {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
    __builtin_nontemporal_store(f32x4{a[0] * s, a[1] * s, b[0] * s, b[1] * s}, reinterpret_cast<f32x4*>(p));
  }
}

// One wavefront per (block, kv-head), all loads issued before the first store.  Keys:
// four dims of a token a lane.  Values: squares of 4 dims x 4 tokens, transposed in
// registers; the 16 lanes of a square's four tokens store 128 contiguous bytes (bf16)
// of a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_read_kernel(T* __restrict__ k_out, T* __restrict__ v_out,
                                                       Kv8Args a) {
  constexpr int LT = D / 4;          // lanes of a token's keys
  constexpr int NK = kBlock * LT / 64;
  constexpr int SQ = D / 64;         // squares of a lane
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i = (int64_t)blockIdx.x * 4 + w;
  const int64_t slot = i / a.hkv;
  if (slot >= a.slots) return;
  const int h = int(i - slot * a.hkv);
  const BlockRows b = find_rows(a, int(slot));
  if (b.off0 == b.off1 || b.id < 0 || b.id >= a.num_blocks) return;
  const int64_t bh = (int64_t)b.id * a.hkv + h;
  const uint8_t* kb = a.kc + bh * (kBlock * D);
  const uint8_t* vb = a.vc + bh * (kBlock * D);
  const float sk = pow2(int(a.scales[2 * bh]) - kExpBias);
  const float sv = pow2(int(a.scales[2 * bh + 1]) - kExpBias);
  auto has = [&](int o) { return o >= b.off0 && o < b.off1; };
  const int kd = 4 * (lane % LT), ko = lane / LT;      // of load 0; 64 / LT tokens a load
  const int vd = 4 * (lane / 4), vo = 4 * (lane % 4);  // of square 0; 64 dims a square

  uint32_t k[NK], v[SQ][4];
#pragma unroll
  for (int u = 0; u < NK; ++u)
    k[u] = *reinterpret_cast<const uint32_t*>(kb + kd / 64 * 1024 + (u * (64 / LT) + ko) * 64 + kd % 64);
#pragma unroll
  for (int sq = 0; sq < SQ; ++sq)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      v[sq][x] = *reinterpret_cast<const uint32_t*>(vb + (64 * sq + vd + x) * kBlock + vo);
#pragma unroll
  for (int u = 0; u < NK; ++u) {
    const int o = u * (64 / LT) + ko;
    if (has(o)) store4(k_out + (int64_t)(b.row0 + o - b.off0) * a.k_stride + (int64_t)h * D + kd, k[u], sk);
  }
#pragma unroll
  for (int sq = 0; sq < SQ; ++sq) {
    transpose4(v[sq]);
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (has(vo + x))
        store4(v_out + (int64_t)(b.row0 + vo + x - b.off0) * a.v_stride + (int64_t)h * D + 64 * sq + vd, v[sq][x], sv);
  }
}

// Slots of n rows of n_seqs sequences: one per row where that is fewer than two per
// sequence and one per 16 rows (decode and verification steps).
Kv8Args with_slots(Kv8Args a) {
  a.slots = int64_t(a.n_tokens) / kBlock + 2 * int64_t(a.n_seqs);
  a.by_token = a.n_tokens <= a.slots;
  if (a.by_token) a.slots = a.n_tokens;
  return a;
}

}  // namespace

int launch_kv8_append(const void* kn, int64_t k_stride, const void* vn, int64_t v_stride,
                      const int32_t* bt, int32_t max_blocks, const int32_t* seq_lens,
                      const int32_t* cu, int32_t n_seqs, int32_t n, void* kc, void* vc,
                      uint8_t* scales, int32_t nb, int32_t hkv, int32_t d, int32_t dtype,
                      hipStream_t stream) {
  const Kv8Args a = with_slots({bt, seq_lens, cu, static_cast<uint8_t*>(kc), static_cast<uint8_t*>(vc), scales,
                  k_stride, v_stride, max_blocks, n_seqs, n, nb, hkv, 0, false});
  const int64_t grid = (a.slots * hkv + 3) / 4;  // a wavefront per (block, kv-head)
  if (grid > INT32_MAX || a.slots > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
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
  const Kv8Args a = with_slots({bt, seq_lens, cu, static_cast<uint8_t*>(const_cast<void*>(kc)),
                  static_cast<uint8_t*>(const_cast<void*>(vc)), const_cast<uint8_t*>(scales),
                  k_stride, v_stride, max_blocks, n_seqs, n, nb, hkv, 0, false});
  const int64_t grid = (a.slots * hkv + 3) / 4;
  if (grid > INT32_MAX || a.slots > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
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
