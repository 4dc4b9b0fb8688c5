// Eviction: of each sequence and kv-head the first F tokens, the last W and the heaviest of
// the rest stay, B in all; their keys, values and weights move together, in order.
//
// Two launches.  The first finds the tokens: a workgroup per (sequence, kv-head) finds the
// (B - F - W)-th largest weight digit by digit (histograms in LDS of 11, 11 and 10 bits of
// the weights' bits, ordered as the numbers are), then writes the positions of what stays
// in order, of equal weights the first ones.  The second moves: a wavefront per block of 16
// tokens that are kept.  Kept tokens only move towards the front: token i comes from a
// position of i or more.  In place, a block is therefore written once every block before it
// and itself have been read: a workgroup takes 16 blocks at a time and waits between.
#include <type_traits>

#include "device_common.h"

namespace pa {
namespace dev {
namespace {

struct EvictArgs {
  const float* w;
  float* w_out;
  int64_t w_stride;
  const int32_t* bt;
  const int32_t* bt_new;
  const int32_t* seq_lens;
  const int32_t* new_lens;
  const int32_t* first;  // or NULL
  int32_t* kept;
  int64_t kept_stride;
  uint8_t* kc;
  uint8_t* vc;
  uint8_t* scales;
  int32_t max_blocks, max_new, window, num_blocks, hkv, groups;
};

constexpr int kMostTokens = 1 << 30;  // of a sequence: positions and their shares fit 32 bits

struct Lens {
  int len, keep, front, window;  // keep 0: nothing to do
};

// A sequence's lengths; one that does not fit the arrays is left alone.
__device__ __forceinline__ Lens lens_of(const EvictArgs& a, int r) {
  const int L = a.seq_lens[r], B = min(a.new_lens[r], L);
  if (B <= 0 || L > kMostTokens || L > a.w_stride || L > int64_t(a.max_blocks) * kBlock || B > a.kept_stride ||
      B > int64_t(a.max_new) * kBlock)
    return {L, 0, 0, 0};
  const int F = a.first ? min(max(a.first[r], 0), B) : 0;
  return {L, B, F, min(a.window, B - F)};
}

// Order of the numbers, as unsigned: NaN last, zeros of either sign alike.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return ~0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kHeld = 16;  // weights of a thread that stay in registers

// NT threads (256 where rows of weights are short: its barriers are cheaper).  A wavefront
// takes an even share of the positions, 64 at a time; up to 16 NT of them are read once, all
// loads issued together, further ones in each pass again, as many at a time.  Bound by its
// passes one after the other (atomics on LDS, the scan of 2048 counts, barriers), not by bytes:
// 8 kv-heads of 16 contexts of 6000-16000 tokens 18 us for 8.6 MB, 33 with the weights read in
// each pass; of 64 contexts of 1000-2000, with 256 threads, 12, 15; an eviction from one 4-bit
// context of 45000 tokens 61, 72 with the further ones read one by one, 67 with 32 NT held,
// which costs one of 6000 17 -> 21.
template <int NT>
__global__ __launch_bounds__(NT) void evict_select_kernel(EvictArgs a) {
  constexpr int kWaves = NT / 64, kBinsPer = 2048 / NT;
  __shared__ int hist[3][2048];
  __shared__ int part[2][kWaves];
  __shared__ int found[3][2];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = blockIdx.x / a.hkv;
  const Lens n = lens_of(a, r);
  if (n.keep == 0) return;
  const float* w = a.w + blockIdx.x * a.w_stride;
  float* out = a.w_out + blockIdx.x * a.w_stride;
  int32_t* kept = a.kept + blockIdx.x * a.kept_stride;
  const int lo = n.front, hi = n.len - n.window;  // candidates
  const int want = n.keep - n.front - n.window;
  const int share = (n.len + NT - 1) / NT * 64;
  const int p0 = min(wv * share, n.len), p1 = min(p0 + share, n.len);

  // A candidate's order, 0 (less than that of any number) for other positions.
  auto order = [&](int i, float x) { return i >= lo && i < hi && i < p1 ? order_of(x) : 0u; };
  float held[kHeld];
  uint32_t orders[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) held[k] = w[max(min(p0 + 64 * k + lane, p1 - 1), 0)];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) orders[k] = order(p0 + 64 * k + lane, held[k]);
  // f(position, weight, order) for the wavefront's positions, 64 at a time
  auto each = [&](auto f) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (p0 + 64 * k < p1) f(p0 + 64 * k + lane, held[k], orders[k]);
    for (int i = p0 + 64 * kHeld; i < p1; i += 64 * kHeld) {
      float x[kHeld];
#pragma unroll
      for (int k = 0; k < kHeld; ++k) x[k] = w[min(i + 64 * k + lane, p1 - 1)];
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (i + 64 * k < p1) f(i + 64 * k + lane, x[k], order(i + 64 * k + lane, x[k]));
    }
  };

  // The want-th largest candidate T, and how many of those equal to it stay.
  uint32_t T = 0;
  int ties = 0;
  if (want > 0) {
    for (int i = tid; i < 3 * 2048; i += NT) hist[i / 2048][i % 2048] = 0;
    __syncthreads();
    int left = want;
    uint32_t prefix = 0, known = 0;  // T's bits found so far, and which
    constexpr int kShift[3] = {21, 10, 0}, kMask[3] = {2047, 2047, 1023};
#pragma unroll
    for (int d = 0; d < 3; ++d) {
      each([&](int, float, uint32_t u) {
        if (u != 0 && (u & known) == prefix) atomicAdd(&hist[d][u >> kShift[d] & kMask[d]], 1);
      });
      __syncthreads();
      // Counts from the largest digit down, kBinsPer of them a thread.
      int h[kBinsPer], mine = 0;
#pragma unroll
      for (int q = 0; q < kBinsPer; ++q) {
        h[q] = hist[d][2047 - kBinsPer * tid - q];
        mine += h[q];
      }
      int sum = mine;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const int o = __shfl_up(sum, m, 64);
        if (lane >= m) sum += o;
      }
      if (lane == 63) part[d & 1][wv] = sum;
      __syncthreads();
      int before = sum - mine;
      for (int v = 0; v < wv; ++v) before += part[d & 1][v];
      // the digit where the count reaches `left`
      if (before < left && before + mine >= left) {
#pragma unroll
        for (int q = 0; q < kBinsPer; ++q) {
          if (before < left && before + h[q] >= left) found[d][0] = 2047 - kBinsPer * tid - q, found[d][1] = left - before;
          before += h[q];
        }
      }
      __syncthreads();
      prefix |= uint32_t(found[d][0]) << kShift[d];
      known |= uint32_t(kMask[d]) << kShift[d];
      left = found[d][1];
    }
    T = prefix;
    ties = left;
  }

  // How many of a wavefront's positions stay, and how many equal T.
  // 0: goes, 1: equals T, 2: stays
  auto kind = [&](int i, uint32_t u) {
    if (u == 0) return i < p1 ? 2 : 0;  // first and last ones; behind the wavefront's
    if (want <= 0) return 0;
    return u > T ? 2 : u == T ? 1 : 0;
  };
  int stay = 0, equal = 0;
  each([&](int i, float, uint32_t u) {
    const int k = kind(i, u);
    stay += __popcll(__ballot(k == 2));
    equal += __popcll(__ballot(k == 1));
  });
  __syncthreads();  // the last digit's counts have been read
  if (lane == 0) part[0][wv] = stay, part[1][wv] = equal;
  __syncthreads();
  int at = 0, eq = 0;  // kept, and equal ones, before this wavefront's
  for (int v = 0; v < wv; ++v) {
    at += part[0][v] + max(0, min(part[1][v], ties - eq));
    eq += part[1][v];
  }
  const uint64_t below = (uint64_t(1) << lane) - 1;
  each([&](int i, float x, uint32_t u) {
    const int k = kind(i, u);
    const uint64_t e = __ballot(k == 1);
    const bool keep = k == 2 || (k == 1 && eq + __popcll(e & below) < ties);
    const uint64_t m = __ballot(keep);
    if (keep) {
      const int to = at + __popcll(m & below);
      kept[to] = i;
      if (w != out) out[to] = x;
    }
    at += __popcll(m);
    eq += __popcll(e);
  });
  if (w != out) return;
  __syncthreads();
  // In place, NT weights are read before they are written.
  for (int i0 = 0; i0 < n.keep; i0 += NT) {
    const int i = i0 + tid;
    float x = 0.f;
    if (i < n.keep) x = w[kept[i]];
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(x) : : "memory");
    __syncthreads();
    if (i < n.keep) out[i] = x;
  }
}

// One block's kept tokens on their way: 16 tokens of a (sequence, kv-head), NS slices from
// slice s0 on: keys and values of 32 dims each; of the 4-bit cache (ELEM 0; else a value's
// bytes) slice 0 is the keys and scales, slice 1 the values.
template <int D, int ELEM, int NS>
struct Moved {
  static constexpr bool KV4 = ELEM == 0;
  static constexpr int kHeadBytes = KV4 ? kBlock * D / 2 : kBlock * D * ELEM;
  static constexpr int kScaleRows = D / 32 + 1;
  static constexpr int U = KV4 ? D / 32 : 2 * ELEM;  // 16-byte units of a token's (32 dims') key
  static constexpr int NK = KV4 ? 1 : U * kBlock / 64;  // loads of a slice's keys
  typedef typename std::conditional<ELEM == 4, uint32_t, uint16_t>::type T;
  struct alignas(16) Half { T x[kBlock / 2]; };      // 8 tokens of a dim
  u32x4 k[KV4 ? 1 : NS][NK];
  u32x4 v4;                     // KV4: dims 32 c + i and 32 c + 16 + i
  Half v[KV4 ? 1 : NS];         // lane (dim, half): dim 32 s + lane % 32
  uint32_t s[2];                // KV4: scale bytes

  // pos: old position of the block's token lane % 16.
  __device__ __forceinline__ void load(const EvictArgs& a, int g, int s0, int pos, const int32_t* bt, int lane) {
    const int id = clamp_block(bt[pos / kBlock], a.num_blocks);
    auto block_of = [&](int o) { return (int64_t)__shfl(id, o, 64) * a.hkv + g; };
    auto off_of = [&](int o) { return __shfl(pos, o, 64) % kBlock; };
    if constexpr (KV4) {
      if (NS > 1 || s0 == 0) {
        const int o = lane / U % kBlock;
        k[0][0] = ld16(a.kc + block_of(o) * kHeadBytes + off_of(o) * (D / 2) + lane % U * 16);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int u = min(64 * i + lane, kScaleRows * kBlock - 1), so = u % kBlock;
          s[i] = a.scales[block_of(so) * (kScaleRows * kBlock) + u / kBlock * kBlock + off_of(so)];
        }
      }
      if (NS > 1 || s0 == 1) {
        v4 = zero16();
#pragma unroll
        for (int t = 0; t < kBlock; ++t) {
          // The token's block, two dims of all its tokens a lane: neighbouring tokens find it
          // in the cache (64 requests, 32000 tokens moved, 28 us; loads of the halves that
          // hold the token 44, all 16 loads before the first use 29).
          const int64_t b = (int64_t)__builtin_amdgcn_readlane(id, t) * a.hkv + g;
          const int off = __builtin_amdgcn_readlane(pos, t) % kBlock;
          const u32x4 x = ld16(a.vc + b * kHeadBytes + 16 * (lane % (D / 2)));
          const uint32_t c0 = (off < 8 ? x[0] : x[1]) >> (4 * (off & 7)) & 15;
          const uint32_t c1 = (off < 8 ? x[2] : x[3]) >> (4 * (off & 7)) & 15;
          v4[t / 8] |= c0 << (4 * (t & 7));
          v4[2 + t / 8] |= c1 << (4 * (t & 7));
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const int u = 64 * i + lane, o = u / U;
        const uint8_t* p = a.kc + block_of(o) * kHeadBytes + key_slot_pos(off_of(o)) * (32 * ELEM) + u % U * 16;
#pragma unroll
        for (int n = 0; n < NS; ++n) k[n][i] = ld16(p + (s0 + n) * (kBlock * 32 * ELEM));
      }
#pragma unroll
      for (int t = 0; t < kBlock / 2; ++t) {
        const int o = lane / 32 * (kBlock / 2) + t;
        const T* p = reinterpret_cast<const T*>(a.vc + block_of(o) * kHeadBytes) + (32 * s0 + lane % 32) * kBlock + off_of(o);
#pragma unroll
        for (int n = 0; n < NS; ++n) v[n].x[t] = p[32 * n * kBlock];
      }
    }
  }

  // The first `count` tokens, to block `id`.
  __device__ __forceinline__ void store(const EvictArgs& a, int g, int s0, int id, int count, int lane) const {
    const int64_t b = (int64_t)id * a.hkv + g;
    if constexpr (KV4) {
      if (NS > 1 || s0 == 0) {
        if (lane < kBlock * U && lane / U < count) st16(a.kc + b * kHeadBytes + lane * 16, k[0][0]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int u = 64 * i + lane;
          if (u < kScaleRows * kBlock && u % kBlock < count) a.scales[b * (kScaleRows * kBlock) + u] = uint8_t(s[i]);
        }
      }
      if ((NS > 1 || s0 == 1) && lane < D / 2) {
        u32x4* p = reinterpret_cast<u32x4*>(a.vc + b * kHeadBytes) + lane;
        u32x4 x = v4;
        if (count < kBlock) {
          const u32x4 was = *p;
          const uint64_t m = (uint64_t(1) << (4 * count)) - 1;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t mi = uint32_t(m >> (32 * (i & 1)));
            x[i] = (x[i] & mi) | (was[i] & ~mi);
          }
        }
        *p = x;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const int u = 64 * i + lane, o = u / U;
        uint8_t* p = a.kc + b * kHeadBytes + key_slot_pos(o) * (32 * ELEM) + u % U * 16;
        if (o < count) {
#pragma unroll
          for (int n = 0; n < NS; ++n) st16(p + (s0 + n) * (kBlock * 32 * ELEM), k[n][i]);
        }
      }
      const int first = lane / 32 * (kBlock / 2);
      T* p = reinterpret_cast<T*>(a.vc + b * kHeadBytes) + (32 * s0 + lane % 32) * kBlock + first;
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        if (count >= first + kBlock / 2) {
          *reinterpret_cast<Half*>(p + 32 * n * kBlock) = v[n];
        } else {
#pragma unroll
          for (int t = 0; t < kBlock / 2; ++t)
            if (first + t < count) p[32 * n * kBlock + t] = v[n].x[t];
        }
      }
    }
  }
};

// To other blocks: one workgroup per four blocks; bound by the caches' lines, of which values
// are read whole, since a dim's 16 tokens lie together (16 contexts of 6000-16000 bf16 tokens
// to a quarter: 520 MB read, 176 written, 150 us, 4.6 TB/s).  In place: one per (sequence, kv-head),
// which takes 16 blocks at a time, or, SLICED, per slice of it: slices do not wait for each
// other.  Sliced is faster while the workgroups do not fill the chip (one context of 16000
// tokens to a quarter, 8 kv-heads, 300 -> 107 us, 16 of 11000 tokens 325 -> 201), and slower
// where they do (64 of 1500 tokens over the 4-bit cache 40 -> 50).
template <int D, int ELEM, bool IN_PLACE, bool SLICED = false>
__global__ __launch_bounds__(IN_PLACE ? 1024 : 256) void evict_move_kernel(EvictArgs a) {
  constexpr int kWaves = IN_PLACE ? 16 : 4;
  constexpr int kAll = ELEM == 0 ? 2 : D / 32, kSlices = SLICED ? kAll : 1, NS = SLICED ? 1 : kAll;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int x = IN_PLACE ? blockIdx.x / kSlices : blockIdx.x / a.groups;
  const int s0 = SLICED ? blockIdx.x - x * kSlices : 0;
  const int r = x / a.hkv, g = x - r * a.hkv;
  const Lens n = lens_of(a, r);
  if (n.keep == 0) return;
  const int32_t* kept = a.kept + x * a.kept_stride;
  const int32_t* bt = a.bt + (int64_t)r * a.max_blocks;
  const int32_t* to = a.bt_new + (int64_t)r * a.max_new;
  const int blocks = (n.keep + kBlock - 1) / kBlock;
  // Where all tokens stay, blocks that are in both tables hold what they have to already, and
  // may be other sequences' too: they are not written.
  if (IN_PLACE && n.keep == n.len) return;
  const int first = n.front / kBlock + (IN_PLACE ? 0 : (blockIdx.x - x * a.groups) * kWaves);
  for (int b0 = first; b0 < (IN_PLACE ? blocks : min(blocks, first + kWaves)); b0 += kWaves) {
    const int b = b0 + wv, count = min(kBlock, n.keep - b * kBlock);
    if (!IN_PLACE && n.keep == n.len && count > 0 && to[b] == bt[b]) continue;
    Moved<D, ELEM, NS> m;
    int id = -1;
    if (count > 0) {
      m.load(a, g, s0, kept[b * kBlock + min(lane % kBlock, count - 1)], bt, lane);
      id = to[b];
    }
    if constexpr (IN_PLACE) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    }
    if (id >= 0 && id < a.num_blocks) m.store(a, g, s0, id, count, lane);
  }
}

}  // namespace

int launch_kv_evict(const float* w, float* w_out, int64_t w_stride, const int32_t* bt,
                    int32_t max_blocks, const int32_t* bt_new, int32_t max_new,
                    const int32_t* seq_lens, const int32_t* new_lens, const int32_t* first,
                    int32_t window, int32_t n_seqs, void* kc, void* vc, uint8_t* scales,
                    int32_t num_blocks, int32_t hkv, int32_t d, int32_t elem, int32_t* kept,
                    int64_t kept_stride, bool in_place, hipStream_t stream) {
  EvictArgs a{w, w_out, w_stride, bt, bt_new, seq_lens, new_lens, first, kept, kept_stride,
              static_cast<uint8_t*>(kc), static_cast<uint8_t*>(vc), scales, max_blocks, max_new, window,
              num_blocks, hkv, 0};
  const int64_t heads = int64_t(n_seqs) * hkv;
  const int64_t blocks = min((kept_stride + kBlock - 1) / kBlock, int64_t(max_new));
  const int64_t groups = (blocks + 3) / 4;
  const bool narrow = w_stride <= 16 * 256;
  // A launch has fewer than 2^32 work-items.  Both launches' are looked at before the first: the
  // selection may write the new weights over the old ones, and a move would then not follow.
  const int64_t threads = max(int64_t(narrow ? 256 : 1024), in_place ? int64_t(1024) : 256 * groups);
  if (heads > UINT32_MAX / threads) return static_cast<int>(hipErrorInvalidValue);
  a.groups = int32_t(groups);
  if (narrow)
    hipLaunchKernelGGL(evict_select_kernel<256>, dim3(unsigned(heads)), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(evict_select_kernel<1024>, dim3(unsigned(heads)), dim3(1024), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || groups == 0) return static_cast<int>(e);
  const bool sliced = heads < 512;
#define PA_MOVE(DD, EE)                                                                              \
  if (in_place && sliced)                                                                            \
    hipLaunchKernelGGL((evict_move_kernel<DD, EE, true, true>), dim3(unsigned(heads * (EE == 0 ? 2 : DD / 32))), \
                       dim3(1024), 0, stream, a);                                                    \
  else if (in_place)                                                                                 \
    hipLaunchKernelGGL((evict_move_kernel<DD, EE, true>), dim3(unsigned(heads)), dim3(1024), 0, stream, a); \
  else                                                                                               \
    hipLaunchKernelGGL((evict_move_kernel<DD, EE, false>), dim3(unsigned(heads * groups)), dim3(256), 0, stream, a)
#define PA_MOVE_D(EE)          \
  if (d == 128) {              \
    PA_MOVE(128, EE);          \
  } else {                     \
    PA_MOVE(64, EE);           \
  }
  switch (elem) {
    case 0: PA_MOVE_D(0); break;
    case 2: PA_MOVE_D(2); break;
    default: PA_MOVE_D(4); break;
  }
#undef PA_MOVE_D
#undef PA_MOVE
  return static_cast<int>(hipGetLastError());
}

}  // namespace dev
}  // namespace pa
