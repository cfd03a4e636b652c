// Rows in pages: written as they come, in 8 bits where the cache holds FP8, and
// read back.
//
// Row r of sequence s is slot r % page of page table[s][r / page], K and V
// [n_pages][hkv][page][d].  An FP8 row x is held as E4M3 codes c and one exponent:
//   e = the least with max |x_i| <= 448 2^e over the finite x_i,   c_i = e4m3(x_i 2^-e),
// so that a row's values keep four significant bits (a power of two costs an
// E4M3 value nothing but range: the smallest values lose at most one of its 18
// binades) and the way back, c_i 2^e, is exact in bf16.  With 448 = 7/8 2^9 and
// max |x| = m 2^k, 1 <= m < 2: e = k - 8 + (m > 7/4).  The byte kept is e + 127.
//
// HBM bound: every row is read once and written once, in pieces of 16 bytes a
// lane (32 of a row on its way into E4M3); a workgroup takes some 16 consecutive tokens of one
// head, which of a prompt lie side by side in their page.  8191 tokens of 8 heads of 128
// in E4M3: 11.6 us written (4.4 TB/s, read plus written), 11.1 us read (4.6 TB/s).  A head's tokens before the next head's took
// 15.4 us written; two, four and eight rows a lane, all requested before the first is used, as long as one in E4M3
// (93, 93 and 96 us for 32768 tokens written and read, one row 92) and longer in bf16.
#include <type_traits>

#include "fdkv_common.h"
#include "fp8.h"
#include "rows_kernels.h"

namespace fdkv {

namespace {

enum : int { kF32 = 0, kBf16 = 1, kC8 = 2 };
constexpr int kThreads = 256;

// Maximum over aligned groups of N lanes; every lane gets its group's.
template <int N>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  auto from = [](uint32_t v, auto ctrl) { return as_u32(dpp<decltype(ctrl)::value>(as_f32(v))); };
  if constexpr (N >= 2) x = max(x, from(x, std::integral_constant<int, kDppQuadXor1>{}));
  if constexpr (N >= 4) x = max(x, from(x, std::integral_constant<int, kDppQuadXor2>{}));
  if constexpr (N >= 8) x = max(x, from(x, std::integral_constant<int, kDppRowHalfMirror>{}));
  if constexpr (N >= 16) x = max(x, from(x, std::integral_constant<int, kDppRowMirror>{}));
  return x;
}

// Slot of a token's row in the pool (page * hkv * page_size ...), or -1: it has none.
__device__ __forceinline__ int64_t slot_of(const PageParams& pg, const int32_t* seqs, const int32_t* rows, int tok, int head) {
  const int seq = seqs ? seqs[tok] : tok, row = rows[tok];
  if ((uint32_t)seq >= (uint32_t)pg.batch || row < 0 || (row >> pg.log_page) >= pg.max_pages) return -1;
  const int id = pg.table[(int64_t)seq * pg.max_pages + (row >> pg.log_page)];
  if ((uint32_t)id >= (uint32_t)pg.n_pages) return -1;
  return (((int64_t)id * pg.hkv + head) << pg.log_page) + (row & ((1 << pg.log_page) - 1));
}

template <int D, int TY, bool WRITE>
__global__ __launch_bounds__(kThreads) void page_rows_kernel(PageRowsParams P) {
  constexpr int E = TY == kF32 ? 4 : 2;
  constexpr int N = WRITE && TY == kC8 ? 2 : 1;              // 16-byte pieces of a lane
  constexpr int LPR = D * E / 16 / N, RPW = kThreads / LPR;  // lanes of a row, rows of a workgroup
  const int r = threadIdx.x / LPR, j = threadIdx.x % LPR;
  // the heads of 16 tokens follow each other, so that the workgroups at work together read a projection's rows whole
  const uint32_t tile = P.by_heads.div(blockIdx.x);
  const int h = (int)(blockIdx.x - tile * 2 * P.pg.hkv);
  const int64_t tok = (int64_t)tile * RPW + r;
  const bool is_v = h >= P.pg.hkv;
  const int head = is_v ? h - P.pg.hkv : h;
  if (tok >= P.n_tokens) return;  // (the lanes of a row leave together)
  uint4* mine = reinterpret_cast<uint4*>(static_cast<uint8_t*>(is_v ? P.rows_v : P.rows_k) + tok * (is_v ? P.v_tok : P.k_tok) +
                                         head * (is_v ? P.v_head : P.k_head)) + j * N;
  uint4 w{}, w2{};
  if constexpr (WRITE) w = *mine;  // (on its way while the row's place is looked up)
  if constexpr (N == 2) w2 = mine[1];
  const int64_t slot = slot_of(P.pg, P.seqs, P.rows, (int)tok, head);
  uint8_t* pool = static_cast<uint8_t*>(is_v ? P.pg.v : P.pg.k);
  if constexpr (TY != kC8) {
    if (slot < 0) return;
    uint4* held = reinterpret_cast<uint4*>(pool) + slot * LPR + j;
    if constexpr (WRITE)
      *held = w;
    else
      *mine = *held;
  } else {
    uint8_t* exps = is_v ? P.pg.v_exp : P.pg.k_exp;
    if constexpr (WRITE) {
      const uint32_t x[8] = {w.x, w.y, w.z, w.w, w2.x, w2.y, w2.z, w2.w};
      // bf16 magnitudes compare as their bits; what is not finite is left out (and held as NaN)
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t lo = x[i] & 0x7FFFu, hi = (x[i] >> 16) & 0x7FFFu;
        top = max(top, max(lo >= 0x7F80u ? 0u : lo, hi >= 0x7F80u ? 0u : hi));
      }
      top = group_max<LPR>(top);
      // top = m 2^k, k + 127 its exponent bits; m > 7/4: fraction bits above 1100000
      const int b = max((int)(top >> 7) - 8 + ((top & 0x7Fu) > 0x60u ? 1 : 0), 1);  // 1 .. 247
      const float f = as_f32((uint32_t)(254 - b) << 23);                            // 2^-(b - 127)
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(bf16_lo(x[2 * i]) * f, bf16_hi(x[2 * i]) * f, 0, false);
        c[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(bf16_lo(x[2 * i + 1]) * f, bf16_hi(x[2 * i + 1]) * f, lo, true);
      }
      if (slot < 0) return;
      reinterpret_cast<uint4*>(pool)[slot * LPR + j] = make_uint4(c[0], c[1], c[2], c[3]);
      if (j == 0) exps[slot] = (uint8_t)b;
    } else {
      if (slot < 0) return;
      const uint2 c = reinterpret_cast<const uint2*>(pool)[slot * LPR + j];
      const float f = as_f32((uint32_t)exps[slot] << 23);
      auto two = [&](uint32_t y, auto hi) {
        typedef float f32x2v __attribute__((ext_vector_type(2)));
        const f32x2v x = __builtin_amdgcn_cvt_pk_f32_fp8((int)y, decltype(hi)::value);
        return cvt_bf16x2(x[0] * f, x[1] * f);
      };
      *mine = make_uint4(two(c.x, std::false_type{}), two(c.x, std::true_type{}), two(c.y, std::false_type{}), two(c.y, std::true_type{}));
    }
  }
}

template <int D, int TY, bool WRITE>
hipError_t launch(PageRowsParams P, hipStream_t s) {
  constexpr int rpw = kThreads / (D * (TY == kF32 ? 4 : 2) / 16) * (WRITE && TY == kC8 ? 2 : 1);
  P.by_heads.set((uint32_t)(2 * P.pg.hkv));
  const dim3 grid((unsigned)(((int64_t)P.n_tokens + rpw - 1) / rpw * (2 * P.pg.hkv)));
  hipLaunchKernelGGL((page_rows_kernel<D, TY, WRITE>), grid, dim3(kThreads), 0, s, P);
  return hipGetLastError();
}

template <bool WRITE>
hipError_t launch_any(const PageRowsParams& P, hipStream_t s) {
  const int ty = !P.pg.bf16 ? kF32 : P.pg.coef8 ? kC8 : kBf16;
  if (P.pg.d == 128) return ty == kF32 ? launch<128, kF32, WRITE>(P, s) : ty == kBf16 ? launch<128, kBf16, WRITE>(P, s) : launch<128, kC8, WRITE>(P, s);
  return ty == kF32 ? launch<64, kF32, WRITE>(P, s) : ty == kBf16 ? launch<64, kBf16, WRITE>(P, s) : launch<64, kC8, WRITE>(P, s);
}

}  // namespace

hipError_t launch_page_write(const PageRowsParams& P, hipStream_t s) { return P.n_tokens ? launch_any<true>(P, s) : hipSuccess; }
hipError_t launch_page_read(const PageRowsParams& P, hipStream_t s) { return P.n_tokens ? launch_any<false>(P, s) : hipSuccess; }

}  // namespace fdkv
