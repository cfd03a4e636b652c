// The index of sparse decode: per channel the least and the largest key of every
// block of 64 tokens, and the selection of the blocks that a decode step reads.
//
// key_bounds: lo[c] = min_t K[t][c], hi[c] = max_t K[t][c] over a block's tokens.
// HBM bound (the keys are read once, a 32nd of them written).  A wave takes a
// block: all of its loads are in flight at once, the two extremes stay in
// registers, and the rows of a load meet in a few lane exchanges.
//
// block_select: for query head g of a KV head's group and block j
//   U_gj = sum_c max(q_c lo_jc, q_c hi_jc) = sum_c q_c (q_c > 0 ? hi_jc : lo_jc),
// the largest logit (before its scale) that a key within the block's bounds can
// have.  A block's rank is max_g (U_gj - max_j U_gj), how near it comes to the
// best block of any of the group's heads, so every head's best block leads.  The
// n_first first and n_last last blocks and the best others are selected, n_sel in
// all, ties to the lower block.  U is summed in fp64, where a product of two stored
// values is exact and a sum of d of them off by at most d 2^-53 sum_c |q_c| max(|lo_jc|, |hi_jc|):
// blocks nearer to each other than that may change places.  Blocks whose bounds agree
// wherever U reads them are equal to the bit, as every block's sum takes the same
// order.  (As q mid + |q| rad, with half the sum and half the difference of the
// bounds, the unread bound's rounding broke such ties; it spares the choice, 0.6 us
// of a 17.3 us call of 2048 blocks for eight heads a group and nothing of the 8.0 us
// of 512 blocks for four.)
//
// Two launches.  block_scores splits the blocks over workgroups (memory bound).
// block_choose, one workgroup per (sequence, KV head), finds the rank of the last
// selected block by one histogram of the ranks between the worst and the best
// (they are differences of one scale, so equal bins spread them) and an exact
// comparison of the ranks in the bin that holds it; only where that bin holds
// more than kChooseList ranks (many equal ones) does a digit by digit selection
// over their bit patterns follow.  Its last pass writes the selected blocks in
// ascending order.
#include "fdkv_common.h"
#include "serving_kernels.h"

namespace fdkv {

namespace {

__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// ---------------------------------------------------------------- bounds
template <int D, bool BF16>
__global__ __launch_bounds__(256) void key_bounds_kernel(BoundsParams P) {
  constexpr int N = BF16 ? 8 : 4;        // channels of a 16-byte piece
  constexpr int NP = D / N;              // pieces of a row
  constexpr int RPL = 64 / NP;           // rows of a load
  constexpr int NL = kBlockTokens / RPL; // loads of a block
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int blk = blockIdx.x * 4 + wave, head = blockIdx.y, layer = blockIdx.z;
  const int t0 = blk * kBlockTokens;
  if (t0 >= P.seq_len) return;
  const int pc = lane % NP, rg = lane / NP;
  const uint4* src = static_cast<const uint4*>(P.k[layer]) + (uint64_t)head * P.seq_len * NP;
  uint4 v[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i)  // rows past the sequence repeat its last one
    v[i] = src[(uint64_t)min(t0 + i * RPL + rg, P.seq_len - 1) * NP + pc];
  float lo[N], hi[N];
#pragma unroll
  for (int i = 0; i < NL; ++i)
#pragma unroll
    for (int c = 0; c < N; ++c) {
      const uint32_t w = word_of(v[i], BF16 ? c / 2 : c);
      const float x = BF16 ? ((c & 1) ? bf16_hi(w) : bf16_lo(w)) : as_f32(w);
      lo[c] = i ? fminf(lo[c], x) : x;
      hi[c] = i ? fmaxf(hi[c], x) : x;
    }
#pragma unroll
  for (int o = NP; o < 64; o *= 2)
#pragma unroll
    for (int c = 0; c < N; ++c) {
      lo[c] = fminf(lo[c], __shfl_xor(lo[c], o, 64));
      hi[c] = fmaxf(hi[c], __shfl_xor(hi[c], o, 64));
    }
  if (rg < 2) {  // rows 0 and 1 of the lanes write the two rows
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = rg ? hi[BF16 ? 2 * i : i] : lo[BF16 ? 2 * i : i];
      if constexpr (BF16)
        w[i] = cvt_bf16x2(a, rg ? hi[2 * i + 1] : lo[2 * i + 1]);  // a key's own value: exact
      else
        w[i] = as_u32(a);
    }
    uint4* dst = static_cast<uint4*>(P.out[layer]) + (((uint64_t)head * P.cap + blk) * 2 + rg) * NP + pc;
    *dst = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ---------------------------------------------------------------- scores
// Lane exchanges of fp64 values without LDS: DPP within rows of 16 lanes, permlane swaps across them.
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
// The two halves that a swap of 16 (32) lanes pairs up, in either order.
template <int N, class F>
__device__ __forceinline__ double swap_f64(double x, F f) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)u, hi = (uint32_t)(u >> 32);
  if constexpr (N == 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), b = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    return f(__builtin_bit_cast(double, ((uint64_t)b[0] << 32) | a[0]), __builtin_bit_cast(double, ((uint64_t)b[1] << 32) | a[1]));
  } else {
    const auto a = __builtin_amdgcn_permlane32_swap(lo, lo, false, false), b = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    return f(__builtin_bit_cast(double, ((uint64_t)b[0] << 32) | a[0]), __builtin_bit_cast(double, ((uint64_t)b[1] << 32) | a[1]));
  }
}
// f over aligned groups of N lanes; every lane gets its group's value.
template <int N, class F>
__device__ __forceinline__ double group_f64(double x, F f) {
  if constexpr (N >= 2) x = f(x, dpp_f64<kDppQuadXor1>(x));
  if constexpr (N >= 4) x = f(x, dpp_f64<kDppQuadXor2>(x));
  if constexpr (N >= 8) x = f(x, dpp_f64<kDppRowHalfMirror>(x));
  if constexpr (N >= 16) x = f(x, dpp_f64<kDppRowMirror>(x));
  if constexpr (N >= 32) x = swap_f64<16>(x, f);
  if constexpr (N >= 64) x = swap_f64<32>(x, f);
  return x;
}
struct AddF64 {
  __device__ __forceinline__ double operator()(double a, double b) const { return a + b; }
};
struct MaxF64 {
  __device__ __forceinline__ double operator()(double a, double b) const { return fmax(a, b); }
};
struct MinF64 {
  __device__ __forceinline__ double operator()(double a, double b) const { return fmin(a, b); }
};

template <int D, int G, bool BF16>
__global__ __launch_bounds__(256) void block_scores_kernel(SelectParams P) {
  constexpr int N = BF16 ? 8 : 4;
  constexpr int NP = D / N;              // lanes of a block, a piece each
  constexpr int BPW = 64 / NP;           // blocks that a wave takes at once
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int sh = blockIdx.y, seq = sh / P.hkv, head = sh - seq * P.hkv;
  const int T = min(max(P.seq_lens[seq], 0), P.max_seq_len);
  const int nb = (T + kBlockTokens - 1) / kBlockTokens;
  const int base = blockIdx.x * kScoreBlocks;
  if (base >= nb) return;
  const int pc = lane % NP, rg = lane / NP;
  const uint4* src = static_cast<const uint4*>(P.bounds) + (uint64_t)sh * P.cap * 2 * NP;
  constexpr int IT = kScoreBlocks / (4 * BPW) > 0 ? kScoreBlocks / (4 * BPW) : 1;
  uint4 lo[IT], hi[IT];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const uint64_t j = min(base + (i * 4 + wave) * BPW + rg, nb - 1);
    lo[i] = src[(j * 2) * NP + pc];
    hi[i] = src[(j * 2 + 1) * NP + pc];
  }
  uint4 qv[G];
#pragma unroll
  for (int g = 0; g < G; ++g)
    qv[g] = static_cast<const uint4*>(P.q)[((uint64_t)seq * P.hq + (uint64_t)head * G + g) * NP + pc];
  auto chan = [](const uint4& v, int c) -> float {
    const uint32_t w = word_of(v, BF16 ? c / 2 : c);
    return BF16 ? ((c & 1) ? bf16_hi(w) : bf16_lo(w)) : as_f32(w);
  };
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int j = base + (i * 4 + wave) * BPW + rg;
    double acc[G];
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g] = 0.0;
#pragma unroll
    for (int c = 0; c < N; ++c) {
      const double l = (double)chan(lo[i], c), h = (double)chan(hi[i], c);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float q = chan(qv[g], c);
        acc[g] = fma((double)q, q > 0.f ? h : l, acc[g]);
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g] = group_f64<NP>(acc[g], AddF64{});
    if (j < nb && pc == 0) {
#pragma unroll
      for (int g = 0; g < G; ++g) P.ws[((uint64_t)sh * G + g) * P.cap + j] = acc[g];
    }
  }
}

// ---------------------------------------------------------------- choice
// (Eight waves: 512 blocks of a sequence 5.2 us, 256 4.8; sixteen, with more to exchange and to wait for, 6.1 and 5.9.  At
// 2048 blocks both take 11.)
constexpr int kChooseThreads = 512;
constexpr int kChooseWaves = kChooseThreads / 64;
constexpr int kChooseBins = 512;
constexpr int kChooseList = 512;
static_assert(kChooseWaves >= 8, "a wave for every query head of a group");
static_assert(kChooseList <= kChooseThreads && kChooseThreads >= 256, "a rank of the list, and a digit, a thread");

constexpr int kChooseHeld = 4096;  // ranks that a workgroup keeps in LDS (32 KB)

// A rank as an unsigned number of the same order.
__device__ __forceinline__ uint64_t order_of(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);  // -0 as +0
  return (u >> 63) ? ~u : u | (1ull << 63);
}

// HELD: the ranks stay in LDS (sequences of at most 4096 blocks), else in the first head's scores.
template <int G, bool HELD>
__global__ __launch_bounds__(kChooseThreads) void block_choose_kernel(SelectParams P) {
  __shared__ double held[HELD ? kChooseHeld : 1];
  __shared__ double red[kChooseWaves];
  __shared__ uint32_t hist[kChooseBins];
  __shared__ uint64_t list[kChooseList];
  __shared__ uint32_t wsum[2][kChooseWaves];
  __shared__ uint32_t s_bin, s_need, s_count, s_n, s_take;
  __shared__ uint64_t s_key;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int sh = blockIdx.x, seq = sh / P.hkv;
  const int T = min(max(P.seq_lens[seq], 0), P.max_seq_len);
  const int nb = (T + kBlockTokens - 1) / kBlockTokens;
  int32_t* out = P.blocks + (uint64_t)sh * P.n_sel;
  const int n = min(P.n_sel, nb);
  if (tid == 0) P.counts[sh] = n;
  for (int i = n + tid; i < P.n_sel; i += kChooseThreads) out[i] = -1;
  if (nb <= P.n_sel) {
    for (int i = tid; i < nb; i += kChooseThreads) out[i] = i;
    return;
  }
  // more blocks than are selected: n_first + n_last <= n_sel < nb, so the two ends are apart
  const int first = P.n_first, last = nb - P.n_last;           // candidates are [first, last)
  const uint32_t need = (uint32_t)(n - P.n_first - P.n_last);  // of them
  double* sc = P.ws + (uint64_t)sh * G * P.cap;
  double* rank = HELD ? held : sc;

  // Every head's best block: 8 / G waves a head (a reduction of every head in every wave would cost G times its
  // instructions).
  constexpr int WPH = kChooseWaves / G;
  double mine[G];  // the thread's first block, requested with the others
#pragma unroll
  for (int g = 0; g < G; ++g) mine[g] = tid < nb ? sc[(uint64_t)g * P.cap + tid] : -INFINITY;
  {
    const double* one = sc + (uint64_t)(wave / WPH) * P.cap;
    double x = -INFINITY;
#pragma unroll 4
    for (int j = (wave % WPH) * 64 + lane; j < nb; j += WPH * 64) x = fmax(x, one[j]);
    x = group_f64<64>(x, MaxF64{});
    if (lane == 0) red[wave] = x;
  }
  hist[tid] = 0;
  if (tid == 0) {
    s_n = s_count = 0;
    s_key = ~0ull;
    s_take = 0;
  }
  __syncthreads();
  double m[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    m[g] = red[g * WPH];
#pragma unroll
    for (int w = 1; w < WPH; ++w) m[g] = fmax(m[g], red[g * WPH + w]);
  }

  // the ranks (every thread keeps its blocks), and the worst finite one
  double worst = 0.0;
  for (int j = tid; j < nb; j += kChooseThreads) {
    double r = -INFINITY;
#pragma unroll
    for (int g = 0; g < G; ++g) r = fmax(r, (j == tid ? mine[g] : sc[(uint64_t)g * P.cap + j]) - m[g]);
    rank[j] = r;
    if (j >= first && j < last && r > -INFINITY) worst = fmin(worst, r);
  }
  worst = group_f64<64>(worst, MinF64{});
  __syncthreads();  // red is read above
  if (lane == 0) red[wave] = worst;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kChooseWaves; ++w) worst = fmin(worst, red[w]);
  // bins of equal width, the best ranks first; any scale keeps the order
  const double scale = worst < 0.0 ? (double)(kChooseBins - 1) / -worst : 0.0;
  auto bin_of = [&](double r) -> uint32_t {
    if (!(r > -INFINITY)) return kChooseBins - 1;
    const double x = -r * scale;
    return x >= (double)(kChooseBins - 1) ? kChooseBins - 1 : (uint32_t)x;
  };
  for (int j = tid; j < nb; j += kChooseThreads)  // (its own blocks: no barrier since they were written)
    if (j >= first && j < last) atomicAdd(&hist[bin_of(rank[j])], 1u);
  __syncthreads();
  // the bin of the need-th best: a running sum over the bins, one a thread
  {
    static_assert(kChooseBins == kChooseThreads, "one bin a thread");
    const uint32_t c = hist[tid];
    uint32_t x = c;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const uint32_t y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    if (lane == 63) wsum[0][wave] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kChooseWaves; ++w) x += w < wave ? wsum[0][w] : 0u;
    if (need > 0 && x >= need && x - c < need) {
      s_bin = (uint32_t)tid;
      s_need = need - (x - c);
      s_count = c;
    }
  }
  __syncthreads();
  // the order of the last selected candidate, and how many of that very order are selected
  if (need > 0) {
    const uint32_t cut = s_bin, in_bin = s_count, left = s_need;
    if (in_bin <= kChooseList) {
      for (int j = tid; j < nb; j += kChooseThreads)
        if (j >= first && j < last && bin_of(rank[j]) == cut) list[atomicAdd(&s_n, 1u)] = order_of(rank[j]);
      __syncthreads();
      if (tid < (int)in_bin) {
        const uint64_t o = list[tid];
        uint32_t above = 0, same = 0;
        for (uint32_t i = 0; i < in_bin; ++i) {
          above += list[i] > o ? 1u : 0u;
          same += list[i] == o ? 1u : 0u;
        }
        if (above < left && above + same >= left) {  // equal ranks all write the same
          s_key = o;
          s_take = left - above;
        }
      }
    } else {
      uint64_t key = 0, mask = 0;
      uint32_t want = left;
      for (int shift = 56; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < nb; j += kChooseThreads) {
          const double r = rank[j];
          const uint64_t o = order_of(r);
          if (j >= first && j < last && bin_of(r) == cut && (o & mask) == key) atomicAdd(&hist[(o >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (tid == 0) {
          uint32_t sum = 0;
          int d = 255;
          while (d > 0 && sum + hist[d] < want) sum += hist[d--];
          s_bin = (uint32_t)d;
          s_need = want - sum;
        }
        __syncthreads();
        key |= (uint64_t)s_bin << shift;
        mask |= 255ull << shift;
        want = s_need;
        __syncthreads();
      }
      if (tid == 0) {
        s_key = key;
        s_take = want;
      }
    }
  }
  __syncthreads();
  const uint64_t key = s_key;
  const uint32_t take = s_take;

  // The selected blocks, ascending: those above `key`, the ends, and the first `take` equal to it.  A block's place is
  // the number of the former before it and of the latter, up to `take`.
  uint32_t above = 0, equal = 0;  // in the chunks before
  for (int j0 = 0; j0 < nb; j0 += kChooseThreads) {
    const int j = j0 + tid;
    const bool live = j < nb, ends = live && (j < first || j >= last);
    const uint64_t o = live ? order_of(rank[j]) : 0;
    const bool gt = ends || (live && need > 0 && o > key), eq = live && !ends && need > 0 && o == key;
    const uint64_t bg = __ballot(gt), be = __ballot(eq);
    if (lane == 0) {
      wsum[0][wave] = (uint32_t)__popcll(bg);
      wsum[1][wave] = (uint32_t)__popcll(be);
    }
    __syncthreads();
    uint32_t g_at = above + (uint32_t)__popcll(bg & ((1ull << lane) - 1)), e_at = equal + (uint32_t)__popcll(be & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < kChooseWaves; ++w) {
      const uint32_t a = wsum[0][w], e = wsum[1][w];
      g_at += w < wave ? a : 0u;
      e_at += w < wave ? e : 0u;
      above += a;
      equal += e;
    }
    const uint32_t at = g_at + min(e_at, take);
    if ((gt || (eq && e_at < take)) && at < (uint32_t)n) out[at] = j;
    if (j0 + kChooseThreads < nb) __syncthreads();
  }
}

template <int D, int G>
hipError_t launch_select_dg(const SelectParams& P, hipStream_t s) {
  const dim3 grid((unsigned)((P.cap + kScoreBlocks - 1) / kScoreBlocks), (unsigned)(P.batch * P.hkv));
  if (P.cap > P.n_sel) {  // otherwise every block of every sequence is selected
    if (P.bf16)
      hipLaunchKernelGGL((block_scores_kernel<D, G, true>), grid, dim3(256), 0, s, P);
    else
      hipLaunchKernelGGL((block_scores_kernel<D, G, false>), grid, dim3(256), 0, s, P);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 units((unsigned)(P.batch * P.hkv));
  if (P.cap <= kChooseHeld)
    hipLaunchKernelGGL((block_choose_kernel<G, true>), units, dim3(kChooseThreads), 0, s, P);
  else
    hipLaunchKernelGGL((block_choose_kernel<G, false>), units, dim3(kChooseThreads), 0, s, P);
  return hipGetLastError();
}

template <int D>
hipError_t launch_select_d(const SelectParams& P, hipStream_t s) {
  switch (P.hq / P.hkv) {
    case 1: return launch_select_dg<D, 1>(P, s);
    case 2: return launch_select_dg<D, 2>(P, s);
    case 4: return launch_select_dg<D, 4>(P, s);
    default: return launch_select_dg<D, 8>(P, s);
  }
}

}  // namespace

hipError_t launch_key_bounds(const BoundsParams& P, hipStream_t s) {
  const int nb = (P.seq_len + kBlockTokens - 1) / kBlockTokens;
  const dim3 grid((unsigned)((nb + 3) / 4), (unsigned)P.hkv, (unsigned)P.n_layers);
  if (nb == 0) return hipSuccess;
  if (P.d == 128) {
    if (P.bf16)
      hipLaunchKernelGGL((key_bounds_kernel<128, true>), grid, dim3(256), 0, s, P);
    else
      hipLaunchKernelGGL((key_bounds_kernel<128, false>), grid, dim3(256), 0, s, P);
  } else {
    if (P.bf16)
      hipLaunchKernelGGL((key_bounds_kernel<64, true>), grid, dim3(256), 0, s, P);
    else
      hipLaunchKernelGGL((key_bounds_kernel<64, false>), grid, dim3(256), 0, s, P);
  }
  return hipGetLastError();
}

hipError_t launch_block_select(const SelectParams& P, hipStream_t s) {
  return P.d == 128 ? launch_select_d<128>(P, s) : launch_select_d<64>(P, s);
}

}  // namespace fdkv
