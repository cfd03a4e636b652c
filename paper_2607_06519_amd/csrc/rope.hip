// The rows of a step on their way into the cache: norm of the query and key
// heads, rotation by position, and the exact rows [batch][Hkv][cap][d].
//
// For a row x of d channels (one head of one token):
//   y = x * rsqrt(mean(x^2) + eps) * w      (query and key rows, where w is given)
//   (y_a, y_b) <- (y_a cos t - y_b sin t, y_b cos t + y_a sin t)
// for every pair i < rot / 2, a = i, b = i + rot / 2 (or a = 2i, b = 2i + 1
// interleaved), t = pos[axis(i)] * inv_freq[i].  Everything is computed in fp32
// and rounded once, at the store; the angle is taken in fp64 turns (a position
// of 10^6 times a frequency near 1 leaves fp32 with 0.06 rad of error) and only
// its fractional part goes on in fp32.
//
// HBM bound: every value is read once and written once, and nothing is shared
// but a token's cosines.  A lane holds two 16-byte pieces of a row that pair
// with each other (piece j and piece j + rot / 2), so a rotation never leaves
// the lane and d / 16 lanes (bf16) hold a row; the sum of squares is a DPP sum
// over them.  A workgroup of four waves takes the cosines of its tokens once
// into LDS (one pair of a token a thread), then walks their rows, the next
// row's loads requested before the current one is turned.
#include "fdkv_common.h"
#include "serving_kernels.h"

namespace fdkv {

namespace {

constexpr int kRopeThreads = 256;

template <bool BF16>
struct Piece {  // a 16-byte piece as fp32
  static constexpr int N = BF16 ? 8 : 4;
  float x[N];
  __device__ __forceinline__ void from(const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
      } else {
        x[i] = as_f32(w[i]);
      }
    }
  }
  __device__ __forceinline__ uint4 to() const {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16)
        w[i] = cvt_bf16x2(x[2 * i], x[2 * i + 1]);
      else
        w[i] = as_u32(x[i]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// MANY: a long call (kRopeMany tokens or more).  Its workgroups take all rows of
// kRopeTokens tokens, so a token's cosines are formed once, and its stores pass
// the caches by.  A step's few rows stay in the caches, where its attention reads
// them, and are spread over as many workgroups as they give, each forming its
// token's cosines for itself.  Times (us, normed heads, replayed from a graph, as
// a step's and so), by tokens:
//                                 512          1024          2048          4096          16384
//   32 + 16 heads of 128, bf16    6.3   6.6    11.2   7.7    19.4  13.6    34.0  25.1    122   80
//   32 + 16 heads of 128, fp32    9.2   8.8    15.1  15.1    25.2  22.9    44.2  42.8    161   153
//   8 + 8 heads of 128, bf16      4.5   4.6     5.6   5.4     8.8   6.6    16.1  10.4    54.6  35.8
//   8 + 4 heads of 64, bf16       3.7   3.8     4.4   4.4     6.6   5.0    10.4   7.7    40.2  24.2
//   1 + 2 heads of 64, bf16       4.1   3.7     4.1   3.7     5.7   4.0     9.2   6.0    28.7  16.1
//   2 + 2 heads of 64, fp32       3.4   3.3     4.0   3.7     4.9   4.3     7.6   5.2    24.3  12.4
// so the number of tokens decides, whatever their rows; 256 tokens of the first take 4.9 and 6.2.
// (8191 tokens of the 8B shape, 201 MB read and written, one call after the other:
// 41.2 us, 4.9 TB/s, and with stores through the caches 45.9.)
template <int D, bool BF16, bool INTER, bool MANY>
__global__ __launch_bounds__(kRopeThreads) void rope_append_kernel(RopeParams P) {
  using Pc = Piece<BF16>;
  constexpr int N = Pc::N;              // channels of a piece
  constexpr int NP = D / N;             // pieces of a row
  constexpr int LPR = NP / 2;           // lanes of a row, two pieces each
  constexpr int RPW = kRopeThreads / LPR;
  constexpr int TPW = MANY ? kRopeTokens : 1;  // tokens of a workgroup
  __shared__ float2 turn[TPW][D / 2];

  const int pairs = P.rot / 2;
  const int64_t tok0 = (int64_t)blockIdx.x * TPW;
  const int nt = (int)min((int64_t)TPW, P.n_tokens - tok0);
  const int rows = P.hq + 2 * P.hkv;    // of a token
  const int total = nt * rows, step = RPW * gridDim.y;
  const int j = threadIdx.x % LPR;
  int r = blockIdx.y * RPW + threadIdx.x / LPR;

  // the lane's pieces: j and its partner in the rotated part, neighbours behind it
  const int hp = pairs / N;             // pieces of half the rotated part
  const int pa = j < hp ? j : 2 * hp + 2 * (j - hp), pb = j < hp ? j + hp : pa + 1;

  auto at = [&](int i, int& t, int& h) {
    t = (int)P.by_rows.div((uint32_t)i);
    h = i - t * rows;
  };
  auto fetch = [&](int i, uint4& a, uint4& b) {
    int t, h;
    at(i, t, h);
    const uint8_t* base = static_cast<const uint8_t*>(h < P.hq ? P.q : h < P.hq + P.hkv ? P.k : P.v);
    const int64_t stride = h < P.hq ? P.q_stride : h < P.hq + P.hkv ? P.k_stride : P.v_stride;
    const int hh = h < P.hq ? h : h < P.hq + P.hkv ? h - P.hq : h - P.hq - P.hkv;
    const uint4* src = reinterpret_cast<const uint4*>(base + (tok0 + t) * stride) + hh * NP;
    a = src[pa];
    b = src[pb];
  };

  uint4 ra{}, rb{};
  if (r < total) fetch(r, ra, rb);
  // norm weights of the lane's pieces
  Pc wqa, wqb, wka, wkb;
  if (P.q_norm) {
    wqa.from(static_cast<const uint4*>(P.q_norm)[pa]);
    wqb.from(static_cast<const uint4*>(P.q_norm)[pb]);
  }
  if (P.k_norm) {
    wka.from(static_cast<const uint4*>(P.k_norm)[pa]);
    wkb.from(static_cast<const uint4*>(P.k_norm)[pb]);
  }
  for (int i = threadIdx.x; i < nt * pairs; i += kRopeThreads) {
    const int t = (int)P.by_pairs.div((uint32_t)i), p = i - t * pairs;
    const double turns = (double)P.pos[(int64_t)P.axis[p] * P.n_tokens + tok0 + t] * P.inv_freq[p] * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    turn[t][p] = make_float2(c, s);
  }
  __syncthreads();

  for (; r < total;) {
    const uint4 a0 = ra, b0 = rb;
    const int next = r + step;
    if (next < total) fetch(next, ra, rb);
    int t, h;
    at(r, t, h);
    const int64_t token = tok0 + t;
    const bool is_q = h < P.hq, is_v = h >= P.hq + P.hkv;
    uint4 oa = a0, ob = b0;
    // rows of a wave may differ in kind: the sum of squares runs on all lanes
    Pc a, b;
    a.from(a0);
    b.from(b0);
    if (P.q_norm || P.k_norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) ss = fmaf(a.x[i], a.x[i], fmaf(b.x[i], b.x[i], ss));
      ss = group_sum<LPR>(ss);
      const bool norm = is_q ? P.q_norm != nullptr : !is_v && P.k_norm != nullptr;
      if (norm) {
        const float f = 1.f / sqrtf(ss * (1.f / D) + P.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          a.x[i] *= f * (is_q ? wqa.x[i] : wka.x[i]);
          b.x[i] *= f * (is_q ? wqb.x[i] : wkb.x[i]);
        }
      }
    }
    if (!is_v) {
      if (j < hp) {
        if constexpr (INTER) {
#pragma unroll
          for (int i = 0; i < N / 2; ++i) {
            const float2 ta = turn[t][pa * (N / 2) + i], tb = turn[t][pb * (N / 2) + i];
            const float a1 = a.x[2 * i], a2 = a.x[2 * i + 1], b1 = b.x[2 * i], b2 = b.x[2 * i + 1];
            a.x[2 * i] = a1 * ta.x - a2 * ta.y;
            a.x[2 * i + 1] = a2 * ta.x + a1 * ta.y;
            b.x[2 * i] = b1 * tb.x - b2 * tb.y;
            b.x[2 * i + 1] = b2 * tb.x + b1 * tb.y;
          }
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float2 cs = turn[t][pa * N + i];
            const float x = a.x[i], y = b.x[i];
            a.x[i] = x * cs.x - y * cs.y;
            b.x[i] = y * cs.x + x * cs.y;
          }
        }
      }
      oa = a.to();
      ob = b.to();
    }
    uint4* dst;
    if (is_q) {
      dst = static_cast<uint4*>(P.q_out) + (token * P.hq + h) * NP;
    } else {
      const int seq = P.seqs ? P.seqs[token] : (int)token, row = P.rows[token];
      const bool held = (uint32_t)seq < (uint32_t)P.batch && (uint32_t)row < (uint32_t)P.cap;
      const int hh = is_v ? h - P.hq - P.hkv : h - P.hq;
      dst = held ? static_cast<uint4*>(is_v ? P.v_out : P.k_out) + (((int64_t)seq * P.hkv + hh) * P.cap + row) * NP : nullptr;
    }
    if (dst) {
      if constexpr (MANY) {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        __builtin_nontemporal_store(u32x4{oa.x, oa.y, oa.z, oa.w}, reinterpret_cast<u32x4*>(dst + pa));
        __builtin_nontemporal_store(u32x4{ob.x, ob.y, ob.z, ob.w}, reinterpret_cast<u32x4*>(dst + pb));
      } else {
        dst[pa] = oa;
        dst[pb] = ob;
      }
    }
    r = next;
  }
}

template <int D, bool BF16, bool MANY>
hipError_t launch_many(RopeParams P, hipStream_t s) {
  constexpr int rpw = kRopeThreads / (D / (BF16 ? 8 : 4) / 2);  // rows of a workgroup at once
  const int rows = P.hq + 2 * P.hkv, tpw = MANY ? kRopeTokens : 1;
  P.by_rows.set((uint32_t)rows);
  P.by_pairs.set((uint32_t)(P.rot / 2 > 0 ? P.rot / 2 : 1));
  const dim3 grid((unsigned)(((int64_t)P.n_tokens + tpw - 1) / tpw), MANY ? 1u : (unsigned)((rows + rpw - 1) / rpw));
  if (P.interleaved)
    hipLaunchKernelGGL((rope_append_kernel<D, BF16, true, MANY>), grid, dim3(kRopeThreads), 0, s, P);
  else
    hipLaunchKernelGGL((rope_append_kernel<D, BF16, false, MANY>), grid, dim3(kRopeThreads), 0, s, P);
  return hipGetLastError();
}

template <int D, bool BF16>
hipError_t launch(const RopeParams& P, hipStream_t s) {
  return P.n_tokens >= kRopeMany ? launch_many<D, BF16, true>(P, s) : launch_many<D, BF16, false>(P, s);
}

}  // namespace

hipError_t launch_rope_append(const RopeParams& P, hipStream_t s) {
  if (P.n_tokens == 0) return hipSuccess;
  if (P.d == 128) return P.bf16 ? launch<128, true>(P, s) : launch<128, false>(P, s);
  return P.bf16 ? launch<64, true>(P, s) : launch<64, false>(P, s);
}

}  // namespace fdkv
