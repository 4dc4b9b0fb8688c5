// Norms of queries and keys for each head, and their rotation by position.
//
// y = x / sqrt(mean(x^2) + eps) * w over a head's D dims, then the first rot dims
// turned in pairs by the position's angles (a table of cosines and sines).
// One pass: D / 8 lanes hold a head's row, 16 bytes of bf16 (32 of float32) each,
// the sum of squares is a reduction over them, and pairs that lie in different
// lanes meet through LDS.
#include "device_common.h"

namespace pa {
namespace dev {
namespace {

struct RopeArgs {
  const int32_t* positions;
  const float* cos_sin;
  int64_t q_stride, k_stride;
  int32_t n_tokens, n_positions, rot, hq, hkv;
  float eps;
};

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

template <typename T, int D, bool NORM, bool PAIRS>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const T* q, const T* k, const T* qw,
                                                           const T* kw, T* q_out, T* k_out,
                                                           RopeArgs a) {
  constexpr int LR = D / 8;       // lanes of a row
  constexpr int RW = 256 / LR;    // rows of a workgroup
  __shared__ float sh[RW][D + 4];
  const int tid = threadIdx.x, lr = tid / LR, c = tid % LR;
  const int heads = a.hq + a.hkv;
  const int64_t i = (int64_t)blockIdx.x * RW + lr;
  const int64_t t = i / heads;
  const int h = int(i % heads);
  const int pos = t < a.n_tokens ? a.positions[t] : -1;
  const bool ok = pos >= 0 && pos < a.n_positions;
  const bool key = h >= a.hq;
  float x[8] = {};
  if (ok) {
    get8(key ? k + t * a.k_stride + (int64_t)(h - a.hq) * D + 8 * c : q + t * a.q_stride + (int64_t)h * D + 8 * c, x);
    if constexpr (NORM) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
#pragma unroll
      for (int m = LR / 2; m >= 1; m >>= 1) s += wave_xor(s, m);
      const float inv = 1.f / sqrtf(s / D + a.eps);
      const T* wt = key ? kw : qw;
      float wv[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
      if (wt) get8(wt + 8 * c, wv);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * wv[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) sh[lr][8 * c + e] = x[e];
  __syncthreads();
  if (!ok) return;
  const float* cs = a.cos_sin + (int64_t)pos * a.rot;
  const int half = a.rot / 2;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = 8 * c + e;
    if (d >= a.rot) continue;
    const bool first = PAIRS ? d % 2 == 0 : d < half;
    const int p = PAIRS ? d / 2 : first ? d : d - half;
    const float other = sh[lr][PAIRS ? d ^ 1 : first ? d + half : d - half];
    x[e] = first ? x[e] * cs[p] - other * cs[half + p] : x[e] * cs[p] + other * cs[half + p];
  }
  put8(key ? k_out + (t * a.hkv + h - a.hq) * D + 8 * c : q_out + (t * a.hq + h) * D + 8 * c, x);
}

template <typename T, int D>
int launch_t(const void* q, const void* k, const void* qw, const void* kw, int32_t flags,
             void* q_out, void* k_out, const RopeArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.n_tokens * (a.hq + a.hkv), per = 256 / (D / 8);
  const int64_t grid = (rows + per - 1) / per;
  if (grid > INT32_MAX) return static_cast<int>(hipErrorInvalidValue);
#define PA_ROPE(N, P)                                                                            \
  hipLaunchKernelGGL((qk_norm_rope_kernel<T, D, N, P>), dim3(unsigned(grid)), dim3(256), 0,      \
                     stream, static_cast<const T*>(q), static_cast<const T*>(k),                 \
                     static_cast<const T*>(qw), static_cast<const T*>(kw), static_cast<T*>(q_out), \
                     static_cast<T*>(k_out), a)
  switch (flags) {
    case 0: PA_ROPE(false, false); break;
    case 1: PA_ROPE(true, false); break;
    case 2: PA_ROPE(false, true); break;
    default: PA_ROPE(true, true); break;
  }
#undef PA_ROPE
  return static_cast<int>(hipGetLastError());
}

}  // namespace

int launch_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                        const int32_t* positions, int32_t n, const float* cos_sin,
                        int32_t n_positions, int32_t rot, const void* qw, const void* kw, float eps,
                        int32_t flags, void* q_out, void* k_out, int32_t hq, int32_t hkv, int32_t d,
                        int32_t dtype, hipStream_t stream) {
  const RopeArgs a{positions, cos_sin, q_stride, k_stride, n, n_positions, rot, hq, hkv, eps};
  if (dtype == 1)
    return d == 128 ? launch_t<__bf16, 128>(q, k, qw, kw, flags, q_out, k_out, a, stream)
                    : launch_t<__bf16, 64>(q, k, qw, kw, flags, q_out, k_out, a, stream);
  return d == 128 ? launch_t<float, 128>(q, k, qw, kw, flags, q_out, k_out, a, stream)
                  : launch_t<float, 64>(q, k, qw, kw, flags, q_out, k_out, a, stream);
}

}  // namespace dev
}  // namespace pa
