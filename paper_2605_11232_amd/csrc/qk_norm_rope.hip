// Norms of queries and keys for each head, and their rotation by position.
//
// y = x / sqrt(mean(x^2) + eps) * w over a head's D dims, then the first rot dims
// turned in pairs (a, b) by the position's angles: (a cos - b sin, b cos + a sin),
// which for a dim with partner `o` is x * cos + o * sin with the sine's sign
// folded in; dims behind rot stay: they are selected, as a product with a sine of zero
// would turn an infinity, or a finite dim beside one, into NaN.
//
// One pass over the rows, bound by memory.  D / 8 lanes hold a row, 16 bytes of
// bf16 (32 of float32) each: dims 8 c .. 8 c + 7 of lane c.  A wavefront keeps one
// token's cosines, sines and weights in registers and takes up to U rows at once
// of 64 / (D / 8) heads, all loads issued before the first is used; partners come
// from the lane they are in (half a rotation away), from the same lane (neighbouring
// pairs), or through LDS where half a rotation is no multiple of eight dims.
#include "device_common.h"

namespace pa {
namespace dev {
namespace {

struct RopeArgs {
  const int32_t* positions;
  const float* cos_sin;
  int64_t q_stride, k_stride;
  int32_t n_tokens, n_positions, rot, hq, hkv;
  int32_t waves;  // wavefronts of a token
  float eps;
};

// Where a dim's partner is.
constexpr int kHalfLanes = 0;  // rot / 2 dims away, a multiple of 8: another lane, same element
constexpr int kHalfLds = 1;    // rot / 2 dims away
constexpr int kPairs = 2;      // the neighbouring dim

template <typename T>
__device__ __forceinline__ void get8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 a = as_bf16x8(ld16(p));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(a[i]);
  } else {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
}
template <typename T>
__device__ __forceinline__ void put8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];
    st16(p, __builtin_bit_cast(u32x4, a));
  } else {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
}

template <typename T, int D, bool NORM, int WHERE, int U>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const T* q, const T* k, const T* qw,
                                                           const T* kw, T* q_out, T* k_out,
                                                           RopeArgs a) {
  constexpr int LR = D / 8;     // lanes of a row
  constexpr int HW = 64 / LR;   // heads of a wavefront at a time
  const int lane = threadIdx.x & 63, c = lane % LR, sub = lane / LR;
  const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = wave / a.waves;
  if (t >= a.n_tokens) return;
  const int h0 = int(wave - t * a.waves) * (U * HW) + sub;
  const int heads = a.hq + a.hkv;
  const int pos = a.positions[t];

  // Rows past the last head read it again and store nothing.
  float x[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = min(h0 + u * HW, heads - 1);
    get8(h < a.hq ? q + t * a.q_stride + (int64_t)h * D + 8 * c
                  : k + t * a.k_stride + (int64_t)(h - a.hq) * D + 8 * c, x[u]);
  }
  if (pos < 0 || pos >= a.n_positions) return;
  float cs[8], sn[8];  // of the dims that are turned
  auto turned = [&](int e) { return WHERE == kHalfLanes ? 8 * c < a.rot : 8 * c + e < a.rot; };
  const float* tab = a.cos_sin + (int64_t)pos * a.rot;
  const int half = a.rot / 2;
  if (WHERE == kHalfLanes || (WHERE == kPairs && a.rot % 8 == 0)) {
    // whole chunks are turned, and the table's rows are 16-byte aligned
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = 1.f, sn[e] = 0.f;
    if (8 * c < a.rot) {
      if constexpr (WHERE == kPairs) {
        const f32x4 co = *reinterpret_cast<const f32x4*>(tab + 4 * c);
        const f32x4 si = *reinterpret_cast<const f32x4*>(tab + half + 4 * c);
#pragma unroll
        for (int e = 0; e < 8; ++e) cs[e] = co[e / 2], sn[e] = e % 2 ? si[e / 2] : -si[e / 2];
      } else {
        const bool first = 8 * c < half;
        const float* p = tab + (first ? 8 * c : 8 * c - half);
        get8(p, cs);
        get8(p + half, sn);
#pragma unroll
        for (int e = 0; e < 8; ++e) sn[e] = first ? -sn[e] : sn[e];
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int d = 8 * c + e;
      const bool first = WHERE == kPairs ? d % 2 == 0 : d < half;
      const int p = WHERE == kPairs ? d / 2 : first ? d : d - half;
      cs[e] = turned(e) ? tab[p] : 1.f;
      sn[e] = turned(e) ? tab[half + p] : 0.f;
      sn[e] = first ? -sn[e] : sn[e];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u * HW;
    const bool key = h >= a.hq;
    if constexpr (NORM) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(x[u][e], x[u][e], s);
#pragma unroll
      for (int m = LR / 2; m >= 1; m >>= 1) s += wave_xor(s, m);
      const float inv = 1.f / sqrtf(s / D + a.eps);
      const T* wt = key ? kw : qw;
      float wv[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
      if (wt) get8(wt + 8 * c, wv);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = x[u][e] * inv * wv[e];
    }
    float o[8];
    if constexpr (WHERE == kPairs) {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = x[u][e ^ 1];
    } else if constexpr (WHERE == kHalfLanes) {
      // rows are whole in the wavefront, so lanes stay within their row
      const int to = lane + (8 * c < half ? half / 8 : 8 * c < a.rot ? -(half / 8) : 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __shfl(x[u][e], to, 64);
    } else {
      // a wavefront's own LDS, whose accesses are in order
      __shared__ float sh[4][HW][D];
      float* row = sh[threadIdx.x >> 6][sub];
#pragma unroll
      for (int e = 0; e < 8; ++e) row[8 * c + e] = x[u][e];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int d = 8 * c + e;
        o[e] = row[d < half ? d + half : d < a.rot ? d - half : d];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = turned(e) ? x[u][e] * cs[e] + o[e] * sn[e] : x[u][e];
    if (h < heads)
      put8(key ? k_out + (t * a.hkv + h - a.hq) * D + 8 * c : q_out + (t * a.hq + h) * D + 8 * c, y);
  }
}

template <typename T, int D, int U>
int launch_u(const void* q, const void* k, const void* qw, const void* kw, int32_t flags,
             void* q_out, void* k_out, RopeArgs a, hipStream_t stream) {
  constexpr int HW = 64 / (D / 8);
  a.waves = (a.hq + a.hkv + U * HW - 1) / (U * HW);
  const int64_t grid = ((int64_t)a.n_tokens * a.waves + 3) / 4;
  if (grid > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
#define PA_ROPE(N, P)                                                                            \
  hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, N, P, U>), dim3(unsigned(grid)), dim3(256), 0,   \
                     stream, static_cast<const T*>(q), static_cast<const T*>(k),                 \
                     static_cast<const T*>(qw), static_cast<const T*>(kw), static_cast<T*>(q_out), \
                     static_cast<T*>(k_out), a)
  const bool norm = (flags & 1) != 0;
  if (flags & 2) {
    if (norm) PA_ROPE(true, kPairs);
    else PA_ROPE(false, kPairs);
  } else if (a.rot % 16 == 0) {
    if (norm) PA_ROPE(true, kHalfLanes);
    else PA_ROPE(false, kHalfLanes);
  } else {
    if (norm) PA_ROPE(true, kHalfLds);
    else PA_ROPE(false, kHalfLds);
  }
#undef PA_ROPE
  return static_cast<int>(hipGetLastError());
}

template <typename T, int D>
int launch_t(const void* q, const void* k, const void* qw, const void* kw, int32_t flags,
             void* q_out, void* k_out, const RopeArgs& a, hipStream_t stream) {
  // Two rows a lane, on one load of the angles, once the rows outgrow the caches:
  // 16384 tokens of 32 + 8 heads in bf16 68 us against 83 with one (four: 69), 4096
  // 19.8 and 21.0 (21.3), 2048 even, 64 tokens 3.7 and 3.1 (4.7); head_dim 64, 16384
  // tokens 40.0 and 43.9, 4096 even.  float32 rows fill a lane's loads alone: 8192
  // tokens 65 us with one, 68 with four.
  if constexpr (sizeof(T) == 2) {
    const int64_t rows = (int64_t)a.n_tokens * (a.hq + a.hkv);
    if (rows * D >= int64_t(1) << 24) return launch_u<T, D, 2>(q, k, qw, kw, flags, q_out, k_out, a, stream);
  }
  return launch_u<T, D, 1>(q, k, qw, kw, flags, q_out, k_out, a, stream);
}

}  // namespace

int launch_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                        const int32_t* positions, int32_t n, const float* cos_sin,
                        int32_t n_positions, int32_t rot, const void* qw, const void* kw, float eps,
                        int32_t flags, void* q_out, void* k_out, int32_t hq, int32_t hkv, int32_t d,
                        int32_t dtype, hipStream_t stream) {
  const RopeArgs a{positions, cos_sin, q_stride, k_stride, n, n_positions, rot, hq, hkv, 0, eps};
  if (dtype == 1)
    return d == 128 ? launch_t<__bf16, 128>(q, k, qw, kw, flags, q_out, k_out, a, stream)
                    : launch_t<__bf16, 64>(q, k, qw, kw, flags, q_out, k_out, a, stream);
  return d == 128 ? launch_t<float, 128>(q, k, qw, kw, flags, q_out, k_out, a, stream)
                  : launch_t<float, 64>(q, k, qw, kw, flags, q_out, k_out, a, stream);
}

}  // namespace dev
}  // namespace pa
