// The merge of the records that a decode over parts writes (parts.h):
//   M = max_i m_i,  o = sum_i acc_i 2^(m_i - M) / sum_i l_i 2^(m_i - M)
// per (sequence, query head), over the records of the sequence's own parts and
// those of the shared ones, whose number a head's workgroups leave with the
// records.  One workgroup a query row: half of a wave's lanes (a quarter at
// d = 64) hold a record's d channels, four each, and every group of them folds
// every 8th (16th) record into a running (M, l, o); the groups meet in LDS.
// Bound by the way to memory and back: the records of one row are some 20 KB.
#include "decode_shape.h"
#include "fdkv_common.h"
#include "serving_kernels.h"

namespace fdkv {

namespace {

template <int D, bool BF16>
__global__ __launch_bounds__(256) void parts_merge_kernel(PartsMergeParams P) {
  constexpr int RS = D + 4;
  constexpr int LPR = D / 4, NG = 256 / LPR;  // lanes of a record, groups of them
  constexpr int U = 8;                        // records of a group in flight
  __shared__ float m_lds[NG], l_lds[NG];
  __shared__ __attribute__((aligned(16))) float o_lds[NG][D];
  // The G rows of a (sequence, KV head), whose records lie side by side, on one XCD (workgroups go to the XCDs in turn).
  const uint32_t x = blockIdx.x & 7u, y = blockIdx.x >> 3, unit = (y >> P.g_shift) * 8 + x;
  if (unit >= (uint32_t)(P.batch * P.hkv)) return;
  const uint32_t seq = P.by_hkv.div(unit);
  const int head = (int)(unit - seq * P.hkv), g = (int)y & (P.G - 1);
  const int c4 = threadIdx.x % LPR, rg = threadIdx.x / LPR;
  const uint64_t stride = (uint64_t)P.G * RS;
  const float* base = P.ws + ((uint64_t)seq * P.hkv + head) * P.n_slots_total * stride + (uint64_t)g * RS;
  const int n = P.shared_counts ? P.own_slots + as_const(P.shared_counts)[head] : P.n_slots_total;

  typedef float f32x4 __attribute__((ext_vector_type(4)));
  float M = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = rg; i0 < n; i0 += NG * U) {
    float2 ml[U];
    f32x4 a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* r = base + (uint64_t)min(i0 + u * NG, n - 1) * stride;
      ml[u] = *reinterpret_cast<const float2*>(r + D);
      a[u] = *reinterpret_cast<const f32x4*>(r + 4 * c4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * NG >= n) break;
      const float mn = fmaxf(M, ml[u].x), fo = merge_weight(M, mn), fw = merge_weight(ml[u].x, mn);
      M = mn;
      l = l * fo + ml[u].y * fw;
      o = o * fo + a[u] * fw;
    }
  }
  if (c4 == 0) {
    m_lds[rg] = M;
    l_lds[rg] = l;
  }
  *reinterpret_cast<f32x4*>(&o_lds[rg][4 * c4]) = o;
  __syncthreads();
  if (threadIdx.x < D) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NG; ++i) top = fmaxf(top, m_lds[i]);
    float lt = 0.f, ot = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float w = merge_weight(m_lds[i], top);
      lt = fmaf(w, l_lds[i], lt);
      ot = fmaf(w, o_lds[i][threadIdx.x], ot);
    }
    const float res = lt == 0.f ? 0.f : ot / lt;  // 0: no token at all (a logit that is not a number makes lt NaN)
    const uint64_t at = ((uint64_t)unit * P.G + g) * D + threadIdx.x;
    if constexpr (BF16)
      static_cast<uint16_t*>(P.out)[at] = (uint16_t)f32_to_bf16_bits(res);
    else
      static_cast<float*>(P.out)[at] = res;
  }
}

}  // namespace

hipError_t launch_parts_merge(const PartsMergeParams& P, hipStream_t s) {
  const dim3 grid((unsigned)(P.batch * P.hkv + 7) / 8 * 8 * P.G), block(256);
  if (P.d == 128) {
    if (P.bf16)
      hipLaunchKernelGGL((parts_merge_kernel<128, true>), grid, block, 0, s, P);
    else
      hipLaunchKernelGGL((parts_merge_kernel<128, false>), grid, block, 0, s, P);
  } else {
    if (P.bf16)
      hipLaunchKernelGGL((parts_merge_kernel<64, true>), grid, block, 0, s, P);
    else
      hipLaunchKernelGGL((parts_merge_kernel<64, false>), grid, block, 0, s, P);
  }
  return hipGetLastError();
}

}  // namespace fdkv
