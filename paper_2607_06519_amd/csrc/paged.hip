// Decode attention over pages of exact rows (fdkv_paged_attn):
//   o = softmax(q K^T scale) V
// of one query token a sequence over the rows its table names, the length split
// over workgroups whose (acc, m, l) records a second launch joins with those of
// other tokens of the same sequences (the records of fdkv_decode_partial over a
// compressed prefix, say).
//
// A wave walks tiles of 32 tokens (16 in fp32) of its own; the columns of its
// matrix products are the G query heads of the group:
//   S^T = K Q^T    A: 16 tokens x 32 channels straight from memory in the
//                  operand's layout, B: the queries, kept in registers;
//   softmax        a column lives on the four lanes l, l + 16, l + 32, l + 48; running
//                  max (moved only by more than 2^8) and sum in fp32;
//   O^T += V^T P^T the probabilities are the B operand where they lie, A:
//                  transposed reads of the V tile, which goes through LDS for that.
// 16 tokens lie in one page (a page holds 16 at least), so that half a tile is
// one base address and one bound: a bound that ends with the sequence's last row
// reads zeros behind it, and a page that is none has a bound of no rows.
// E4M3 codes are widened to bf16 (exact); a row's exponent multiplies its logits
// (K) and its probability (V), both exactly.  Probabilities are rounded to bf16
// (2^-8 each at most) for the product, their sum is not.
//
// What bounds it: HBM, behind a start of some 4 us (three trips to memory that need each other: what the launch says;
// length, pages and queries; rows).  131072 tokens of 8 heads of 128 (bf16, 537 MB): 93 us, 5.8 TB/s, and 4.6 for the
// join; 64 sequences of 100 to 8000 tokens 223 us for 1.21 GB, 5.4 TB/s; 32768 tokens in E4M3 (68 MB) 15.5 us, 4.4 TB/s,
// and 4.7.  Two and three tiles in flight a wave instead of one gain nothing, whether one workgroup runs on a CU or
// several (E4M3, us of a pass: 32768 tokens, where a wave walks eight tiles, 314, 315 and 323; 8000 tokens, two tiles a
// wave, 88.8, 93.9 and 95.8; 16 sequences of 1000 to 16000 tokens 485, 501 and 510).
#include "parts.h"
#include "rows_kernels.h"

namespace fdkv {

namespace {

using namespace parts;

template <int D, int TY>
struct Paged {
  using S = TileOf<D, TY>;
  static constexpr bool F32 = TY == kTyF32, C8 = TY == kTyC8;
  static constexpr int RB = D * (F32 ? 4 : 2);       // bytes of a row as operands take it
  static constexpr int HB = C8 ? D : RB;             // bytes of a row in its page
  static constexpr int TI = F32 ? 1 : 2;             // halves of 16 tokens of a tile
  static constexpr int TOK = 16 * TI;
  static constexpr int LJ = HB / 64;                 // 16-byte loads of a lane's row part, a half's K
  static constexpr int LPR = HB / 16, RPL = 64 / LPR, LV = 16 / RPL;  // rowwise: lanes of a row, rows of a load, loads of a half's V
  static constexpr int KK = F32 ? D / 16 : D / 32;   // operand pieces of a row, of a lane
  static constexpr int CT = D / 16;
  static constexpr int TILE_BYTES = TOK * RB;
  static constexpr int MP = D + 4;                   // floats of a row of the merge
  static constexpr int MERGE = 4 * 16 * MP * 4;
  static constexpr int LDS = 4 * TILE_BYTES > MERGE ? 4 * TILE_BYTES : MERGE;
  // Byte of a 16-byte piece of a row of the V tile.  A transposed read takes 32 bytes of each of eight rows at once
  // (fp32: 64 bytes of four rows four apart): the permutation puts them in distinct banks.
  static __device__ __forceinline__ uint32_t at(int row, int piece) {
    const int f = F32 ? ((row >> 2) & 3) << 2 : D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1;
    return (uint32_t)(row * RB + ((piece ^ f) << 4));
  }
};

template <int D, int TY>
__global__ __launch_bounds__(256) void paged_attn_kernel(PagedParams P) {
  using S = Paged<D, TY>;
  constexpr bool F32 = S::F32, C8 = S::C8;
  constexpr int TI = S::TI, TOK = S::TOK, LJ = S::LJ, LV = S::LV, CT = S::CT, KK = S::KK, MP = S::MP, RS = D + 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[S::LDS];
  __shared__ float ml_lds[4][16][2];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lc = lane & 15, lg = lane >> 4;
  const uint32_t y = P.by_hkv.div(blockIdx.x);
  const int head = (int)(blockIdx.x - y * P.pg.hkv);
  const int seq = (int)P.by_chunks.div(y), chunk = (int)(y - seq * P.n_chunks);
  const int hkv = P.pg.hkv, G = 1 << P.g_shift, lp = P.pg.log_page;
  const int c0 = chunk * P.chunk;
  // a length, the pages of the chunk (two a lane) and the queries, requested in one go
  const int page0 = c0 >> lp;
  const int32_t* row = P.pg.table + (int64_t)seq * P.pg.max_pages;
  const int my_page = row[min(page0 + lane, P.pg.max_pages - 1)], my_page2 = row[min(page0 + 64 + lane, P.pg.max_pages - 1)];
  uint4 qf[KK];
  {
    const uint8_t* src = static_cast<const uint8_t*>(P.q) + ((int64_t)seq * P.hq + (int64_t)head * G + min(lc, G - 1)) * S::RB;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qf[kk] = *reinterpret_cast<const uint4*>(src + (C8 ? 128 * (kk / 2) + 32 * lg + 16 * (kk % 2) : 64 * kk + 16 * lg));
  }
  const int T = min(max(as_const(P.lens)[seq], 0), P.max_len);
  const bool single = P.n_chunks == 1 && P.n_more == 0;
  if (c0 >= T && !(single && chunk == 0)) return;  // (the join counts the chunks by the length, too)
  const int end = min(c0 + P.chunk, T);

  // queries: the operand's channels of piece kk are 32 kk + 8 lg .. (E4M3: 64 (kk / 2) + 16 lg + 8 (kk % 2) ..,
  // fp32: 16 kk + 4 lg ..), columns past the group are zero
  auto settle_queries = [&]() __attribute__((always_inline)) {  // (once the first rows are requested)
    const uint32_t keep = lc < G && P.scale_log2 != 0.f ? 0xFFFFFFFFu : 0u;
    const uint32_t sign = P.scale_log2 < 0.f ? (F32 ? 0x80000000u : 0x80008000u) : 0u;  // the largest product is the largest logit
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const uint4 v = qf[kk];
      qf[kk] = make_uint4((v.x ^ sign) & keep, (v.y ^ sign) & keep, (v.z ^ sign) & keep, (v.w ^ sign) & keep);
    }
  };
  const float scale = P.scale_log2 == 0.f ? 1.f : fabsf(P.scale_log2);

  float m = -INFINITY, l = 0.f;
  f32x4_t acc[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  struct Ahead {
    uint4 k[TI][LJ], v[TI][LV];
    uint32_t ke[TI], ve[TI];
    int live[TI];  // rows of the half that count
  };
  const uint32_t k_off = (uint32_t)(lc * S::HB + lg * 16), v_off = (uint32_t)(lane * 16);
  auto load = [&](int t, Ahead& a) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      const int th = t + 16 * i;  // first token of the half
      const int at = min(max((th >> lp) - page0, 0), 127);
      const int id = at < 64 ? __builtin_amdgcn_readlane(my_page, at) : __builtin_amdgcn_readlane(my_page2, at - 64);
      const bool ok = th < end && (uint32_t)id < (uint32_t)P.pg.n_pages;
      a.live[i] = ok ? min(16, end - th) : 0;
      const int64_t slot = ok ? (((int64_t)id * hkv + head) << lp) + (th & ((1 << lp) - 1)) : 0;
      const auto kr = rsrc(static_cast<const uint8_t*>(P.pg.k) + slot * S::HB, (uint64_t)a.live[i] * S::HB);
      const auto vr = rsrc(static_cast<const uint8_t*>(P.pg.v) + slot * S::HB, (uint64_t)a.live[i] * S::HB);
#pragma unroll
      for (int j = 0; j < LJ; ++j) a.k[i][j] = ld128<0>(kr, k_off + 64 * j);
#pragma unroll
      for (int j = 0; j < LV; ++j) a.v[i][j] = ld128<0>(vr, v_off + 1024 * j);
      if constexpr (C8) {  // (a page holds a multiple of 16 rows: the four exponents of a lane's rows lie in it)
        const auto ker = rsrc(P.pg.k_exp + slot, ok ? 16 : 0), ver = rsrc(P.pg.v_exp + slot, ok ? 16 : 0);
        a.ke[i] = __builtin_amdgcn_raw_buffer_load_b32(ker, 4 * lg, 0, 0);
        a.ve[i] = __builtin_amdgcn_raw_buffer_load_b32(ver, 4 * lg, 0, 0);
      }
    }
  };

  uint8_t* vt = lds + wave * S::TILE_BYTES;
  // Tile t from its buffer, which then takes the wave's next one.
  Ahead a;
  auto step = [&](int t) __attribute__((always_inline)) {
    int live[TI];
    uint32_t ke[TI], ve[TI];
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      live[i] = a.live[i];
      ke[i] = a.ke[i];
      ve[i] = a.ve[i];
    }
    // V to LDS
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < LV; ++j) {
        const int row = 16 * i + S::RPL * j + lane / S::LPR, piece = lane % S::LPR;
        const uint4 w = a.v[i][j];
        if constexpr (C8) {
          *reinterpret_cast<uint4*>(vt + S::at(row, 2 * piece)) = widen8(w.x, w.y);
          *reinterpret_cast<uint4*>(vt + S::at(row, 2 * piece + 1)) = widen8(w.z, w.w);
        } else {
          *reinterpret_cast<uint4*>(vt + S::at(row, piece)) = w;
        }
      }
    // logits
    f32x4_t s[TI];
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      s[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        uint4 op;
        if constexpr (C8)
          op = kk % 2 ? widen8(a.k[i][kk / 2].z, a.k[i][kk / 2].w) : widen8(a.k[i][kk / 2].x, a.k[i][kk / 2].y);
        else
          op = a.k[i][kk];
        if constexpr (F32) {
#pragma unroll
          for (int w = 0; w < 4; ++w)
            s[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(as_f32(word(op, w)), as_f32(word(qf[kk], w)), s[i], 0, 0, 0);
        } else {
          s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, op), __builtin_bit_cast(bf16x8_t, qf[kk]), s[i], 0, 0, 0);
        }
      }
    }
    load(t + 4 * TOK, a);  // (behind the end: no rows)

    bool whole = true;
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      if constexpr (C8)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i][r] *= as_f32(((ke[i] >> (8 * r)) & 0xFFu) << 23);
      whole = whole && live[i] == 16;
    }
    if (!whole) {
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (4 * lg + r >= live[i]) {
            s[i][r] = -INFINITY;
            ve[i] &= ~(0xFFu << (8 * r));  // whatever it is: the row's probability is 0
          }
    }
    float mx = s[0][0];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[i][r]);
    mx = scale * col_max(mx);
    if (__any(mx > m + kSlack)) {
      const float mn = fmaxf(m, mx);
      const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[c][r] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    uint32_t pb[4];
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      float p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[r] = __builtin_amdgcn_exp2f(fmaf(s[i][r], scale, -ref));
        l += p[r];
        if constexpr (C8) p[r] *= as_f32(((ve[i] >> (8 * r)) & 0xFFu) << 23);
      }
      if constexpr (F32) {
#pragma unroll
        for (int r = 0; r < 4; ++r) pb[r] = as_u32(p[r]);
      } else {
        pb[2 * i] = cvt_bf16x2(p[0], p[1]);
        pb[2 * i + 1] = cvt_bf16x2(p[2], p[3]);
      }
    }
    // outputs
    lds_fence();
    if constexpr (F32) {
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float v = *reinterpret_cast<const float*>(vt + S::at(4 * lg + r, 4 * c + (lc >> 2)) + (lc & 3) * 4);
          acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, as_f32(pb[r]), acc[c], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        i16x4_t h[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
          h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_i16x4_t*)(vt + S::at(16 * i + 4 * lg + (lc >> 2), 2 * c + ((lc & 3) >> 1)) + (lc & 1) * 8));
        const i16x8_t av = {h[0][0], h[0][1], h[0][2], h[0][3], h[1][0], h[1][1], h[1][2], h[1][3]};
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, av),
                                                         __builtin_bit_cast(bf16x8_t, make_uint4(pb[0], pb[1], pb[2], pb[3])), acc[c], 0, 0, 0);
      }
    }
    lds_fence();
  };
  const int t0 = c0 + TOK * wave;
  if (t0 < end) load(t0, a);
  settle_queries();
  for (int t = t0; t < end; t += 4 * TOK) step(t);
  l = col_sum(l);

  // the waves' sums
  __syncthreads();
  float* o_lds = reinterpret_cast<float*>(lds);  // [4][16][MP]
  if (lc < G) {
    if (lg == 0) {
      ml_lds[wave][lc][0] = m;
      ml_lds[wave][lc][1] = l;
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) *reinterpret_cast<f32x4_t*>(o_lds + (wave * 16 + lc) * MP + 16 * c + 4 * lg) = acc[c];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < G * (D / 4); i += 256) {
    const int g = i / (D / 4), c4 = i % (D / 4);
    float M = -INFINITY, lt = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, ml_lds[w][g][0]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = merge_weight(ml_lds[w][g][0], M);
      lt = fmaf(f, ml_lds[w][g][1], lt);
      o = o + *reinterpret_cast<const f32x4_t*>(o_lds + (w * 16 + g) * MP + 4 * c4) * f;
    }
    if (single) {
      const float inv = lt == 0.f ? 0.f : 1.f / lt;  // 0: no row at all
      const int64_t at = ((int64_t)seq * P.hq + (int64_t)head * G + g) * D + 4 * c4;
      if constexpr (F32)
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(P.out) + at) = o * inv;
      else
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out) + at) = make_uint2(cvt_bf16x2(o[0] * inv, o[1] * inv), cvt_bf16x2(o[2] * inv, o[3] * inv));
    } else {
      float* rec = P.ws + ((((int64_t)seq * hkv + head) * P.n_chunks + chunk) * G + g) * RS;
      *reinterpret_cast<f32x4_t*>(rec + 4 * c4) = o;
      if (c4 == 0) *reinterpret_cast<float2*>(rec + D) = make_float2(M, lt);
    }
  }
}

// Joins the records of a query row: those of the chunks that its length fills, and `more`.  A workgroup takes CH of
// the D channels; a group of CH / 4 lanes folds every NG-th record, the groups meet in LDS.  (One workgroup reads its row's
// records at some 10 GB/s: 86 records of 32 rows take 6.6 us, with 32 channels a workgroup 4.2; 16 records 3.0 and
// 3.3, and 512 rows and more give workgroups enough.)
template <int D, int CH, bool BF16>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedParams P) {
  constexpr int RS = D + 4, LPR = CH / 4, NG = 256 / LPR, U = 4;
  __shared__ float m_lds[NG], l_lds[NG];
  __shared__ __attribute__((aligned(16))) float o_lds[NG][CH];
  const uint32_t row = blockIdx.x / (D / CH);  // (sequence, query head)
  const int part = (int)(blockIdx.x % (D / CH)) * CH;
  const int G = 1 << P.g_shift;
  const uint32_t unit = row >> P.g_shift, seq = P.by_hkv.div(unit);
  const int g = (int)row & (G - 1);
  const int c4 = threadIdx.x % LPR, rg = threadIdx.x / LPR;
  const int T = min(max(as_const(P.lens)[seq], 0), P.max_len);
  const int own = (int)P.by_chunk.div((uint32_t)(T + P.chunk - 1)), n = own + P.n_more;
  const float* base = P.ws + ((int64_t)unit * P.n_chunks * G + g) * RS;
  const float* more = P.more + ((int64_t)unit * P.n_more * G + g) * RS;
  float M = -INFINITY, l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = rg; i0 < n; i0 += NG * U) {
    float2 ml[U];
    f32x4_t a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * NG, n - 1);
      const float* r = i < own ? base + (int64_t)i * G * RS : more + (int64_t)(i - own) * G * RS;
      ml[u] = *reinterpret_cast<const float2*>(r + D);
      a[u] = *reinterpret_cast<const f32x4_t*>(r + part + 4 * c4);
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
  *reinterpret_cast<f32x4_t*>(&o_lds[rg][4 * c4]) = o;
  __syncthreads();
  if (threadIdx.x < CH) {
    float top = -INFINITY, lt = 0.f, ot = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) top = fmaxf(top, m_lds[i]);
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float w = merge_weight(m_lds[i], top);
      lt = fmaf(w, l_lds[i], lt);
      ot = fmaf(w, o_lds[i][threadIdx.x], ot);
    }
    const float res = lt == 0.f ? 0.f : ot / lt;
    const int64_t at = (int64_t)row * D + part + threadIdx.x;
    if constexpr (BF16)
      static_cast<uint16_t*>(P.out)[at] = (uint16_t)f32_to_bf16_bits(res);
    else
      static_cast<float*>(P.out)[at] = res;
  }
}

template <int D, int TY>
hipError_t launch(PagedParams P, hipStream_t s) {
  const int batch = P.pg.batch;
  P.by_hkv.set((uint32_t)P.pg.hkv);
  P.by_chunks.set((uint32_t)P.n_chunks);
  const dim3 grid((unsigned)((int64_t)batch * P.pg.hkv * P.n_chunks));
  hipLaunchKernelGGL((paged_attn_kernel<D, TY>), grid, dim3(256), 0, s, P);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (P.n_chunks == 1 && P.n_more == 0)) return e;
  const unsigned rows = (unsigned)(batch * P.hq);
  P.by_chunk.set((uint32_t)P.chunk);
  if (rows <= 256 && P.n_chunks + P.n_more > 24)
    hipLaunchKernelGGL((paged_join_kernel<D, 32, TY != kTyF32>), dim3(rows * (D / 32)), dim3(256), 0, s, P);
  else
    hipLaunchKernelGGL((paged_join_kernel<D, D, TY != kTyF32>), dim3(rows), dim3(256), 0, s, P);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn(const PagedParams& P, hipStream_t s) {
  const int ty = !P.pg.bf16 ? kTyF32 : P.pg.coef8 ? kTyC8 : kTyBf16;
  if (P.pg.d == 128) return ty == kTyF32 ? launch<128, kTyF32>(P, s) : ty == kTyBf16 ? launch<128, kTyBf16>(P, s) : launch<128, kTyC8>(P, s);
  return ty == kTyF32 ? launch<64, kTyF32>(P, s) : ty == kTyBf16 ? launch<64, kTyBf16>(P, s) : launch<64, kTyC8>(P, s);
}

}  // namespace fdkv
