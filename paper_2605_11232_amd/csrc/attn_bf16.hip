// The attention calls' launches over bf16, 8-bit and 4-bit caches, the items over the bf16
// cache, and the merge of split results.
#include "attn_items.h"

namespace pa {
namespace dev {

extern template int launch_items<8>(const AttnArgs&, int32_t, int32_t, int32_t, hipStream_t,
                                    hipEvent_t, hipEvent_t);
extern template int launch_items<4>(const AttnArgs&, int32_t, int32_t, int32_t, hipStream_t,
                                    hipEvent_t, hipEvent_t);

namespace {

// Combine split partial results by log-sum-exp: one workgroup per four rows (a
// merge group, or a piece of a key-split tile's), half a wavefront per row (32 lanes over the
// output dims, 16-byte partial loads).  The partial outputs of up to 16 parts
// are requested before the part LSEs are reduced, so a row costs about one
// memory round trip; parts are combined in split order (deterministic).  A part
// whose sum is NaN has the log-sum-exp NaN, so that the row comes out NaN.
template <int D>
__global__ __launch_bounds__(kMergeRows * 32) void merge_kernel(AttnArgs a) {
  constexpr int VD = D / 32;  // output dims per lane
  constexpr int C = 16;       // parts whose loads are in flight together
  typedef float vecf __attribute__((ext_vector_type(VD)));
  int narrow = a.merge_narrow;
  if (narrow < 0) {  // an earlier library's plan
    const int n_tmpl = a.plan[H_N_GROUP_TMPL];
    narrow = int(gridDim.x) == n_tmpl ? n_tmpl : a.plan[H_N_GROUP_NARROW];
  }
  const int g = blockIdx.y;
  int t = blockIdx.x, sub = 0;  // template, and which of its rows
  if (t >= narrow) {
    sub = (t - narrow) % kWideGroupParts;
    t = narrow + (t - narrow) / kWideGroupParts;
  }
  const int32_t* gr = a.plan + a.plan[H_GROUP_OFF] + t * kGroupWords;
  const int lr = sub * kMergeRows + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int half = threadIdx.x & 32;  // first lane of this row's half wavefront
  const int nrows = gr[G_NROWS];
  if (sub * kMergeRows >= nrows) return;
  const bool valid = lr < nrows;
  const int r = gr[G_SEQ], row0 = gr[G_ROW0];
  const int nsplit = gr[G_NSPLIT], stride = gr[G_STRIDE];
  // partial row of split 0 (rows past nrows repeat the group's last row, in
  // bounds, and store nothing)
  const int64_t prow = (int64_t)gr[G_PART] + (int64_t)g * a.plan[H_HEAD_PARTIAL] + min(lr, nrows - 1);
  auto part_o = [&](int s) {
    return reinterpret_cast<const vecf*>(a.ws_o + (prow + (int64_t)s * stride) * D) + lane;
  };
  auto part_lse = [&](int s) { return a.ws_lse[prow + (int64_t)s * stride]; };
  vecf x[C];
  auto load_batch = [&](int s0) {
#pragma unroll
    for (int u = 0; u < C; ++u)
      if (s0 + u < nsplit) x[u] = *part_o(s0 + u);
  };
  load_batch(0);
  // max and sum of exp over the part LSEs, 32 parts per round
  const float lse0 = lane < nsplit ? part_lse(lane) : kNegInf;
  float mx = lse0;
  for (int s = 32 + lane; s - lane < nsplit; s += 32) mx = fmaxf(mx, s < nsplit ? part_lse(s) : kNegInf);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
  // Without any finite part both references are 0: all weights are then zero, and
  // the row is zeros, or NaN where the parts hold it.
  const bool none = mx == kNegInf;
  const float ref = none ? 0.f : mx;
  float sum = exp2f((lse0 - ref) * kLog2e);
  for (int s = 32 + lane; s - lane < nsplit; s += 32)
    if (s < nsplit) sum += exp2f((part_lse(s) - ref) * kLog2e);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
  const float lse_v = ref + kLn2 * __log2f(sum);
  const float wref = none ? 0.f : lse_v;
  vecf o_acc = {};
  // weight of part s0 + lane of the current round of 32, held by that lane
  float wl = exp2f((lse0 - wref) * kLog2e);
  for (int s0 = 0; s0 < nsplit; s0 += C) {
    if (s0 > 0) {
      load_batch(s0);
      if (s0 % 32 == 0) {
        const int s = s0 + lane;
        wl = s < nsplit ? exp2f((part_lse(s) - wref) * kLog2e) : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < C; ++u)
      if (s0 + u < nsplit) o_acc += __shfl(wl, half | ((s0 + u) & 31), 64) * x[u];
  }
  if (!valid) return;
  const int qs = a.cu_q[r];
  const int rho = row0 + lr;
  const int qi = rho / a.group;
  const int hq = g * a.group + (rho - qi * a.group);
  __bf16 ob[VD];
#pragma unroll
  for (int k = 0; k < VD; ++k) ob[k] = (__bf16)o_acc[k];
  __bf16* op = a.out + ((int64_t)(qs + qi) * a.hq + hq) * D + VD * lane;
  if constexpr (VD == 4) *reinterpret_cast<u32x2*>(op) = __builtin_bit_cast(u32x2, ob);
  else *reinterpret_cast<uint32_t*>(op) = __builtin_bit_cast(uint32_t, ob);
  // a NaN sum: minus infinity, as where one item writes the row
  if (a.lse && lane == 0) a.lse[(int64_t)(qs + qi) * a.hq + hq] = lse_v == lse_v ? lse_v : kNegInf;
}

}  // namespace

int launch_attn_bf16(const void* q, const void* kc, const void* vc, const uint8_t* scales, int32_t bits, int32_t num_blocks,
                     const int32_t* bt, int32_t max_blocks, const int32_t* seq_lens,
                     const int32_t* cu_q, int32_t hq, int32_t hkv, int32_t d, float scale,
                     const int32_t* plan, int32_t grid, int32_t n_tile, int32_t n_merge,
                     int32_t merge_narrow, bool wide_rows, bool tail, int64_t partial_rows, void* ws, void* out,
                     float* lse, hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  AttnArgs a;
  a.q = static_cast<const __bf16*>(q);
  a.kc = static_cast<const __bf16*>(kc);
  a.vc = static_cast<const __bf16*>(vc);
  a.scales = scales;
  a.bt = bt;
  a.seq_lens = seq_lens;
  a.cu_q = cu_q;
  a.plan = plan;
  a.out = static_cast<__bf16*>(out);
  a.lse = lse;
  a.ws_o = static_cast<float*>(ws);
  a.ws_lse = a.ws_o ? a.ws_o + partial_rows * d : nullptr;
  a.max_blocks = max_blocks;
  a.num_blocks = num_blocks;
  a.hq = hq;
  a.hkv = hkv;
  a.group = hq / hkv;
  a.merge_narrow = merge_narrow;
  a.scale_log2 = scale * kLog2e;
  if (grid > 0) {
    // tiles and rows together: the tile path's register budget holds the
    // wide row path too
    const bool rows = grid > n_tile;
    const int mix = (n_tile == 0 ? (wide_rows ? 6 : 2) : (rows ? 7 : 1)) | (tail ? 8 : 0);
    // the caller's timing events ride on the dispatches (start on the first
    // kernel, stop on the last): no event packets between the kernels
    hipEvent_t stop_here = n_merge > 0 ? nullptr : ev_stop;
    const auto items = bits == 4 ? launch_items<4> : bits == 8 ? launch_items<8> : launch_items<16>;
    const int rc = items(a, d, mix, grid, stream, ev_start, stop_here);
    if (rc) return rc;
  }
  if (n_merge > 0) {
    hipEvent_t start_here = grid > 0 ? nullptr : ev_start;
    if (d == 128)
      hipExtLaunchKernelGGL(merge_kernel<128>, dim3(n_merge / hkv, hkv), dim3(kMergeRows * 32), 0, stream,
                            start_here, ev_stop, 0, a);
    else
      hipExtLaunchKernelGGL(merge_kernel<64>, dim3(n_merge / hkv, hkv), dim3(kMergeRows * 32), 0, stream,
                            start_here, ev_stop, 0, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return static_cast<int>(e);
  }
  if (grid <= 0 && n_merge <= 0) {
    // nothing launched: the events still mark this point of the stream
    for (hipEvent_t ev : {ev_start, ev_stop}) {
      const hipError_t e = ev ? hipEventRecord(ev, stream) : hipSuccess;
      if (e != hipSuccess) return static_cast<int>(e);
    }
  }
  return 0;
}

}  // namespace dev
}  // namespace pa
