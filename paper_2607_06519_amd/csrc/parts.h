// Decode attention over parts (fdkv_decode_parts): whole spans, the selected
// blocks of a span, the exact tail, and spans that all sequences of the batch
// share.  One softmax over all of them: every workgroup writes an (acc, m, l)
// record per query row of its chunk, and the records merge as those of the other
// decode calls do.
//
// The columns of a wave's matrix products are query rows: the G heads of a
// sequence's group, or, over a shared span, 16 NQ rows of the whole batch, so that
// a shared token is read and rebuilt once for all of them.  It walks tiles of TOK =
// 32 tokens (16 in fp32): workgroups of 16 or 32 rows have waves with tiles of their
// own and no barrier before the merge of their records; in those of 64 or 128 rows
// the four waves take 16 NQ rows each of the same tile, which they stage together,
// and two barriers a tile hand it over:
//   S^T = K~ Q^T   A: 16 tokens x 32 channels straight from memory in the
//                  operand's layout (the four waves' tile: from LDS), B: the
//                  queries, kept in registers;
//   softmax        a column lives on the four lanes l, l + 16, l + 32, l + 48, its
//                  logits in their registers; running max (moved only by more
//                  than 2^8) and sum in fp32;
//   O^T += V~^T P^T  the probabilities are the B operand where they lie (the
//                  tokens of a lane's S^T registers are the tokens of its B
//                  slots), A: transposed reads of the V tile, which goes through
//                  LDS for that, its 16-byte pieces permuted by the row
//                  (piece_at).
// K~ = M + R and V~ = M + R: M as stored (bf16 or E4M3 widened to bf16, exact),
// R a tile of LDS that is zero but for the residual entries (or the rows of a
// token-level set) of the tile, each in its place: +-D of a pair is a bf16 value;
// the sum of a block of four's weighted coefficients goes in as its bf16 rounding
// and once more as the rest, so a rebuilt row carries 2^-16 of its residual.  (V's
// rest costs a layer of a shared span of 12345 tokens up to 5% (64 rows: bf16 31.1 and
// 32.6 us, E4M3 29.4 and 29.5; 256 rows of E4M3 54.0 and 54.8), 8% in bf16 at 32 rows
// (23.3 and 25.2), and of selected blocks 2 to 4%.)  R multiplies the same operands as
// M; no rebuilt value is rounded and no entry is gathered per query row.
// Probabilities are rounded to bf16 (2^-8 each at most) for the product, their sum is not: as in the ordinary decode, a
// second term would double the products with V.  Outputs of bf16 queries are 1.6e-3 to 2.0e-3 of their norm off the
// exact ones, of which their own rounding is 1.6e-3 to 1.7e-3.
//
// What bounds it.  Parts of single sequences: HBM where a wave has several tiles (selected blocks of 16 sequences' fp8
// caches, all heads exact: 33.5 us a layer for 135 MB, 4.0 TB/s), else the way to the first one, three trips to memory that need
// each other (what the launch says; lengths, offsets and blocks; rows): 64 blocks of one sequence take 10 us for 18 MB.
// Shared spans: HBM for plain heads, and for residual ones the placing of their entries in R.  16 sequences of four
// heads on 32768 tokens (bf16, pairs of k = 16): 41 us a layer for 161 MB, 3.9 TB/s, tails included (all heads plain 37, residual 50, exact 38); of eight heads
// on 131072 tokens with token-level sets 149 us for 564 MB, 3.8 TB/s, with all heads plain 125 us.
#pragma once

#include <type_traits>

#include "decode_shape.h"
#include "fdkv_common.h"
#include "serving_kernels.h"

namespace fdkv {

namespace parts {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef short i16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;

constexpr uint32_t kOob = 0x80000000u;  // buffer offset past every plane (planes are < 2^31 bytes): loads read 0
constexpr float kSlack = 8.f;           // log2 headroom of the running reference max

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* base, uint64_t bytes) {
  const uint32_t n = bytes > 0xFFFFFFFFull ? 0xFFFFFFFFu : (uint32_t)bytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, n, 0x00020000);
}
template <int CACHE>
__device__ __forceinline__ uint4 ld128(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  const auto v = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, CACHE);
  return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ uint2 ld64(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  const auto v = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
  return make_uint2(v[0], v[1]);
}

template <bool HI>
__device__ __forceinline__ uint32_t e4m3x2_bf16(uint32_t w) {  // exact: every E4M3 value is a bf16 value
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
}
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b) {
  return make_uint4(e4m3x2_bf16<false>(a), e4m3x2_bf16<true>(a), e4m3x2_bf16<false>(b), e4m3x2_bf16<true>(b));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Max / sum over the four lanes of a column (l, l + 16, l + 32, l + 48).
__device__ __forceinline__ float col_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float col_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// What a rounding to `hi` leaves of x; nothing of an infinite one (inf - inf is no number).
__device__ __forceinline__ float rest_of(float x, float hi) { return fabsf(hi) == INFINITY ? 0.f : x - hi; }

// Orders the compiler's LDS accesses; the hardware runs a wave's in order.
__device__ __forceinline__ void lds_fence() { asm volatile("" ::: "memory"); }

enum : int { kTyF32 = 0, kTyBf16 = 1, kTyC8 = 2 };

template <int D, int TY>
struct TileOf {
  static constexpr bool F32 = TY == kTyF32;
  static constexpr int E = F32 ? 4 : 2;            // bytes of an element
  static constexpr int TOK = F32 ? 16 : 32;        // tokens of a tile
  static constexpr int RB = D * E;                 // bytes of a row
  static constexpr int NP = RB / 16;               // 16-byte pieces of a row
  static constexpr int RPL = 64 / NP;              // rows of a load
  static constexpr int NL = D / 16;                // loads of a tile's K (V): TOK * RB / 1024
  static constexpr int KK = F32 ? D / 16 : D / 32; // pieces of the channels in an operand row
  static constexpr int TI = F32 ? 1 : 2;           // 16-token operands of a tile
  static constexpr int TILE_BYTES = TOK * RB;
  static constexpr int CT = D / 16;                // 16-channel tiles of the output
  static constexpr int TPB = kBlockTokens / TOK;   // tiles of a selected block
};

// First of the four tokens of lane group g's rows of the i-th 16-token operand.
// (An E4M3 slot holds rows r and r + 512 / D of a 1 KB block, which go to the two
// operands of one lane; the other types take the same order.)
template <int D, int TY>
__device__ __forceinline__ int quad_row(int g, int i) {
  if constexpr (TY == kTyF32) return 4 * g;
  return D == 128 ? 8 * g + 4 * i : 16 * (g >> 1) + 4 * (g & 1) + 8 * i;
}

// Byte of a 16-byte piece of a row in an LDS tile: pieces permuted so that the
// 16 rows of an operand (one piece of each) lie in distinct banks.  (bf16 rows of
// 128 channels, by counters: reading operands and staging rows have no conflict,
// as reads and writes in a line have none; a transposed read, of two pieces of
// 16 rows, has one for each of its other cycles, 24% of the LDS cycles of a plain
// head.)
template <int D, int TY>
__device__ __forceinline__ uint32_t piece_at(int row, int piece) {
  int f;
  if constexpr (TY == kTyF32)
    f = row & 15;
  else if constexpr (D == 128)
    f = (row & 3) | (((row >> 3) & 3) << 2);
  else
    f = ((row >> 1) & 1) | (((row >> 2) & 1) << 1) | (((row >> 4) & 1) << 2);
  return (uint32_t)(row * TileOf<D, TY>::RB + ((piece ^ f) << 4));
}

// Eight consecutive residual entries of a tile as loaded, and (blocks of four)
// the code before them and the two entries after.
struct Entries {
  uint4 ix;
  uint4 v0, v1;
  uint32_t prev, nix, nv0, nv1;
};

}  // namespace parts

// Residual kinds of a launch: up to eight entries a lane and tile, eight at a time of one token (k a multiple of
// eight); any other number of entries; a token-level set.
enum : int { kFewEntries = 1, kManyEntries = 2, kTokenSet = 3 };

// Workgroups to a CU that the registers have to leave room for.  A spill in the
// walk would wait for every load in flight.
constexpr int parts_per_cu(int KIND, bool q4) { return KIND == kManyEntries && q4 ? 1 : 2; }

// LDS of a workgroup.  A token group's: the V tile, then R with a row behind it that takes what has no place (CG = 4:
// the K tile, and R of K, of V and, of a block of four, of K's and V's rests).
template <int D, int CG, int TY, bool q4>
struct PartsLds {
  using S = parts::TileOf<D, TY>;
  static constexpr bool REST = q4 && !S::F32;  // a residual has a bf16 rest
  static constexpr int RT = S::TILE_BYTES + S::RB;
  static constexpr int GROUP = CG == 1 ? S::TILE_BYTES + RT : 2 * S::TILE_BYTES + (REST ? 4 : 2) * RT;
  static_assert(GROUP % S::RB == 0 && S::TILE_BYTES % S::RB == 0, "tiles start at a multiple of a row");
  static constexpr int MP = D + 4;             // floats of a row of the merge (padded against bank conflicts)
  static constexpr int TILES = 4 / CG * GROUP, MERGE = 4 * 16 * MP * 4;
  static constexpr int BYTES = TILES > MERGE ? TILES : MERGE;
};

// CG column groups of 16 NQ columns each, a wave apiece, by TG = 4 / CG token
// groups: CG = 1, four waves with tiles of their own, or CG = 4, four that walk the
// same tiles.  There each wave stages its share of K and V, one places the residual
// entries of K, one those of V (two more the rests), and two barriers a tile hand
// the tiles over.
template <int D, int NQ, int CG, int TY, int KIND, bool q4>
__device__ __forceinline__ void parts_body(const PartsParams& P, const PartsSide& L, uint32_t w, uint8_t* lds, float (*ml_lds)[16][2]) {
  using namespace parts;
  static_assert(CG == 4 || CG == 1, "the launched forms");
  using S = TileOf<D, TY>;
  constexpr bool F32 = S::F32;
  constexpr int TOK = S::TOK, RB = S::RB, NP = S::NP, RPL = S::RPL, NL = S::NL, KK = S::KK, TI = S::TI, CT = S::CT;
  constexpr int TG = 4 / CG, COLS = 16 * NQ * CG;
  constexpr int RS = D + 4;
  using Lds = PartsLds<D, CG, TY, q4>;
  constexpr bool REST = Lds::REST;
  constexpr int kRt = Lds::RT, kGroupLds = Lds::GROUP, MP = Lds::MP;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % 4, lane = threadIdx.x & 63;
  const int lc = lane & 15, lg = lane >> 4;  // column (or operand row) and lane group
  const int tg = wave / CG, cg = wave % CG;
  // ---- what the launch says, fetched in one go and kept (left to itself the compiler reads it piece by piece, each
  // piece a trip to memory)
  DivU by_slots = L.by_slots, by_hkv = P.by_hkv, by_groups = L.by_groups, by_topk = P.by_topk;
  int hkv = P.hkv, hq = P.hq, G = P.G, g_shift = P.g_shift, n_slots = L.n_slots, tiles_per_wg = L.tiles_per_wg;
  int res_cost = L.res_cost, row_groups = L.row_groups, rows = L.rows, by_cost = L.by_cost, n_blocks = P.n_blocks, block = P.block, slot0 = L.slot0;
  int shared = L.shared, pos = P.pos, nb = P.bsize, k = P.topk, tail_cap = P.tail_cap, n_slots_total = P.n_slots_total;
  const void *q_all = P.q, *tail_k = P.tail_k, *tail_v = P.tail_v;
  float *ws = P.ws, w1 = P.wres[0], w2 = P.wres[1], w3 = P.wres[2], scale_log2 = P.scale_log2;
  PartsPart pt = L.part[0], pt1 = L.part[1];
  int base1 = L.part_base[1], base2 = L.part_base[2];
  asm volatile("" : "+s"(by_slots.mul), "+s"(by_slots.shift), "+s"(by_hkv.mul), "+s"(by_hkv.shift), "+s"(by_groups.mul),
               "+s"(by_groups.shift), "+s"(hkv), "+s"(hq), "+s"(G), "+s"(g_shift), "+s"(n_slots), "+s"(tiles_per_wg),
               "+s"(row_groups), "+s"(rows), "+s"(res_cost), "+s"(by_cost));
  asm volatile("" : "+s"(n_blocks), "+s"(block), "+s"(slot0), "+s"(shared), "+s"(q_all), "+s"(base1), "+s"(base2), "+s"(pt.lens),
               "+s"(pt.cache), "+s"(pt.modes), "+s"(pt.seg_off), "+s"(pt.blocks), "+s"(pt.counts), "+s"(pt.n_sel), "+s"(pt.max_len));
  asm volatile("" : "+s"(pt1.lens), "+s"(pt1.cache), "+s"(pt1.modes), "+s"(pt1.seg_off), "+s"(pt1.blocks), "+s"(pt1.counts),
               "+s"(pt1.n_sel), "+s"(pt1.max_len));
  asm volatile("" : "+s"(ws), "+s"(tail_k), "+s"(tail_v), "+s"(by_topk.mul), "+s"(by_topk.shift), "+s"(pos), "+s"(nb), "+s"(k),
               "+s"(tail_cap), "+s"(n_slots_total), "+s"(w1), "+s"(w2), "+s"(w3), "+s"(scale_log2));

  // ---- which chunk
  int row0 = 0;
  if (shared) {
    // the row groups of one chunk follow each other on one XCD (workgroups go to the XCDs in turn)
    const uint32_t y = w >> 3, ym = by_groups.div(y);
    row0 = (int)(y - ym * row_groups) * COLS;
    w = ym * 8 + (w & 7u);
    if (w >= (uint32_t)(hkv * n_slots)) return;
  }
  const uint32_t sl = by_hkv.div(w);
  int head = (int)(w - sl * hkv), seq = (int)by_slots.div(sl);  // (shared: sequence 0)
  int slot = (int)sl - seq * n_slots, chunk0 = slot, head_slots = 0;
  if (res_cost) {
    // A residual head's tokens take longer and all workgroups run at once, so that the slowest head's would be waited
    // for: the workgroups go to the heads by what their tokens take.  Lane h: head h.
    const uint32_t b = lane < hkv ? pt.modes[block * hkv + lane] : 0u;
    uint32_t c = lane < hkv ? (mode_of(b) == kResidual ? (uint32_t)res_cost : 16u) : 0u;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const uint32_t y = __shfl_up(c, o, 64);
      c += lane >= o ? y : 0u;
    }
    const uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)c, 63);
    const uint32_t end = (uint32_t)(hkv * n_slots) * c / total;  // first workgroup behind head h's
    head = __builtin_popcountll(__ballot(lane < hkv && end <= w));
    const int from = head ? __builtin_amdgcn_readlane((int)end, head - 1) : 0;
    head_slots = __builtin_amdgcn_readlane((int)end, head) - from;
    slot = chunk0 = (int)w - from;
  }
  if (slot >= base1) {
    pt = pt1;
    chunk0 = slot - base1;
    if (slot >= base2) {
      int i = 2;
      while (i + 1 < kMaxParts && slot >= L.part_base[i + 1]) ++i;
      pt = L.part[i];
      chunk0 = slot - L.part_base[i];
    }
  }
  slot += slot0;
  const bool tail = pt.cache == nullptr, picked = pt.n_sel > 0;
  if (by_cost && !tail) {
    // Workgroups w and w + 256 share a CU (where every CU has one before any has two): the first 256 take the heads by
    // rising cost, the next by falling, so that a residual or exact head meets a shared one.  Lane h: head h.
    const uint32_t md = lane < hkv ? (uint32_t)mode_of(pt.modes[((uint64_t)seq * n_blocks + block) * hkv + lane]) : 4u;
    int rank = 0, before = 0;
#pragma unroll
    for (uint32_t c = 0; c < 4; ++c) {
      const uint64_t of = __ballot(md == c);
      rank = md == c ? before + __builtin_popcountll(of & ((1ull << lane) - 1)) : rank;
      before += __builtin_popcountll(of);
    }
    const int place = (sl * hkv >> 8) & 1u ? hkv - 1 - head : head;  // (one order for all heads of the chunk)
    head = __builtin_ctzll(__ballot(lane < hkv && rank == place));
  }

  // ---- queries, requested first (a column past the rows repeats the last one's and is zeroed)
  auto row_of = [&](int col, int& s, int& g) __attribute__((always_inline)) {  // (sequence, head of the group)
    const int r = row0 + col, rc = min(r, rows - 1);
    s = seq + (rc >> g_shift);
    g = rc & (G - 1);
    return r < rows;
  };
  auto q_row = [&](int s, int g) __attribute__((always_inline)) {
    return reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(q_all) + ((uint64_t)s * hq + (uint64_t)head * G + g) * RB);
  };
  uint4 qf[NQ][KK];
  bool q_ok[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    int s, g;
    q_ok[i] = row_of(16 * (cg * NQ + i) + lc, s, g);
    const uint4* src = q_row(s, g);
#pragma unroll
    for (int j = 0; j < KK; ++j) qf[i][j] = src[4 * j + lg];
  }

  // ---- what the unit's arrays say, requested in one go: a length, the mode's word, the segment's offset, the number
  // of selected blocks, and the blocks of the wave's tiles (lane i: tile i).  (What a part has not points to its
  // lengths and is not used.)
  const uint64_t u = tail ? 0 : ((uint64_t)seq * n_blocks + block) * hkv + head;
  const int64_t unit = picked ? (int64_t)seq * hkv + head : 0;
  const auto* words = as_const(reinterpret_cast<const uint32_t*>(pt.modes));
  const auto* offs = as_const(reinterpret_cast<const uint32_t*>(pt.seg_off));
  const int len = as_const(pt.lens)[seq];
  const uint32_t mode_word = words[u >> 2], off_lo = offs[2 * u], off_hi = offs[tail ? 0 : 2 * u + 1];
  const int n_picked = as_const(pt.counts)[unit];
  if (res_cost) tiles_per_wg = ((min(max(len, 0), pt.max_len) + TOK - 1) / TOK + TG * head_slots - 1) / (TG * head_slots) * TG;
  chunk0 *= tiles_per_wg;  // the chunk's first tile
  int my_block = pt.blocks[unit * pt.n_sel + (picked ? min((chunk0 + tg + TG * lane) / S::TPB, pt.n_sel - 1) : 0)];
  asm volatile("" ::"s"(len), "s"(mode_word), "s"(off_lo), "s"(off_hi), "s"(n_picked));
  const int T = min(max(len, 0), pt.max_len);
  const uint32_t mbyte = tail ? (uint32_t)kExact : (mode_word >> (8 * (u & 3))) & 0xFFu;
  const uint64_t seg_off = tail ? 0 : ((uint64_t)off_hi << 32) | off_lo;
  const bool bad_unit = !unit_byte_ok(mbyte, KIND == kTokenSet ? P.n_rates : 0) || (seg_off & (kPlaneAlign - 1));
  const int mode = mode_of(mbyte);
  const int n_tiles = picked && T > 0 ? min(max(n_picked, 0), pt.n_sel) * S::TPB : (T + TOK - 1) / TOK;  // of the part
  if (my_block < 0 || my_block >= (T + kBlockTokens - 1) / kBlockTokens) my_block = -1;
  const int end = min(chunk0 + tiles_per_wg, n_tiles);
  // the wave's tiles: chunk0 + tg + TG i, i < n (CG = 4: the same number for every wave, for the barriers)
  const int n = CG == 1 ? (chunk0 + tg < end ? (end - chunk0 - tg + TG - 1) / TG : 0) : (end - chunk0 + TG - 1) / TG;

  // The scale's sign goes to the queries, so that a column's largest product is its largest logit; a scale of zero
  // zeroes them.  (Once the first tile is requested: the queries were before it.)
  const float scale = scale_log2 == 0.f ? 1.f : fabsf(scale_log2);
  auto settle_queries = [&]() __attribute__((always_inline)) {
    const uint32_t sign = scale_log2 < 0.f ? (F32 ? 0x80000000u : 0x80008000u) : 0u;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const uint32_t keep = q_ok[i] && scale_log2 != 0.f ? 0xFFFFFFFFu : 0u;
#pragma unroll
      for (int j = 0; j < KK; ++j) {
        uint4& v = qf[i][j];
        v = make_uint4((v.x ^ sign) & keep, (v.y ^ sign) & keep, (v.z ^ sign) & keep, (v.w ^ sign) & keep);
      }
    }
  };

  float m[NQ], l[NQ];
  f32x4_t acc[NQ][CT];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    m[q] = -INFINITY;
    l[q] = 0.f;
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[q][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  uint8_t* vt = lds + tg * kGroupLds;                  // the V tile
  uint8_t* kt = vt + S::TILE_BYTES;                    // CG = 4: the K tile
  uint8_t* r_k = kt + (CG == 1 ? 0 : S::TILE_BYTES);   // R of K, of V, of their rests (CG == 1: one after the other)
  uint8_t* r_v = CG == 1 ? r_k : r_k + kRt;
  uint8_t* r_rest = CG == 1 ? r_k : r_k + 2 * kRt;
  uint8_t* r_vrest = CG == 1 ? r_k : r_k + 3 * kRt;
  // CG = 4: the wave's tile of R (0: K, 1: V, 2: K's rest, 3: V's)
  const int role = CG == 1 ? 0 : cg, roles = REST ? 4 : 2;
  uint8_t* rt = r_k + (CG == 1 ? 0 : role < roles ? role : 0) * kRt;
  // Hands LDS tiles from the waves that wrote them to those that read them.
  auto hand_over = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    lds_fence();
  };
  const uint8_t* seg = pt.cache + seg_off;

  // The walk is compiled for each kind of unit, so that every load of a tile is
  // issued unconditionally (a tile that the wave has not takes the out-of-range
  // offset) and the compiler can wait for exactly the loads it needs.  (With the
  // block size and the entries a lane decided at run time it waits for all of them:
  // a residual unit's tile took 11 us.)
  auto walk = [&](auto c8_tag, auto res_tag) __attribute__((always_inline)) {
    constexpr bool C8 = decltype(c8_tag)::value;       // shared planes and residual values in E4M3
    constexpr int RES = decltype(res_tag)::value ? KIND : 0;
    constexpr bool ENT = RES == kFewEntries || RES == kManyEntries, SET = RES == kTokenSet;
    // tiles in flight behind the current one: two where the registers hold them.  (CG = 1 has four tiles of K and V in
    // flight a workgroup as it is, and 32 columns a wave leave no room for a second.)
    constexpr int DEPTH = CG == 4 && NQ == 1 ? 2 : 1;
    constexpr int NCH = RES == kManyEntries ? 2 : 1;   // chunks of eight entries a lane that travel ahead
    constexpr int C = C8 ? 1 : S::E;                   // bytes of a stored coefficient
    constexpr int NLD = C8 ? NL / 2 : NL;              // loads of a tile's K (V)

    // ---- planes
    const uint32_t dense = C8 ? ((uint32_t)T * D + kC8Block - 1) / kC8Block * kC8Block : (uint32_t)T * RB;
    const uint32_t plane = (dense + kPlaneAlign - 1) / kPlaneAlign * kPlaneAlign;
    const uint8_t* kb = seg + (uint64_t)(mode == kExact ? pos : 0) * plane;
    const uint8_t* vb = kb + (uint64_t)(mode == kExact ? nb : 1) * plane;
    if (tail) {
      const uint64_t off = ((uint64_t)seq * hkv + head) * (uint64_t)tail_cap * RB;
      kb = static_cast<const uint8_t*>(tail_k) + off;
      vb = static_cast<const uint8_t*>(tail_v) + off;
    }
    const auto kr = rsrc(kb, dense), vr = rsrc(vb, dense);
    // residual entries
    const uint32_t ib = ENT ? (uint32_t)T * k * (q4 ? 2 : 1) : 0, xb = ENT ? (uint32_t)T * k * C : 0;
    const uint32_t ip = (ib + kPlaneAlign - 1) / kPlaneAlign * kPlaneAlign, xp = (xb + kPlaneAlign - 1) / kPlaneAlign * kPlaneAlign;
    const uint8_t* ent = seg + 2 * (uint64_t)plane;
    // (whole 16-byte pieces: a load whose last word lies half behind the bytes would read 0 for all of it.  The
    // plane's padding may hold anything; entries of tokens behind the last are not used.)
    const uint32_t ibr = (ib + 15) & ~15u, xbr = (xb + 15) & ~15u;
    // (CG = 4: the wave reads the entries of its role, K's or V's, into what is K's buffer here)
    const uint64_t k_at = CG > 1 && (role & 1) ? (uint64_t)ip + xp : 0;
    const uint32_t live = CG > 1 && role >= roles ? 0u : ~0u;
    const auto ikr = rsrc(ent + k_at, ibr & live), xkr = rsrc(ent + k_at + ip, xbr & live);
    const auto ivr = rsrc(ent + ip + xp, ibr), xvr = rsrc(ent + 2 * (uint64_t)ip + xp, xbr);
    // token-level set
    TokLayout L{};
    uint64_t set_bytes = 0;
    if constexpr (SET) {
      const int ppm = unit_ppm(P.res_ppm, P.n_rates, P.rates_ppm, mbyte);
      L = tok_layout(mode, (uint64_t)T, D, ppm, S::E, C, nb);
      set_bytes = residual_token_count((uint64_t)T, ppm) * (uint64_t)(nb - 1) * D * C;
    }
    const auto hkr = rsrc(seg + (CG > 1 && (role & 1) ? L.hv : L.hk), CG > 1 && role >= roles ? 0 : set_bytes);
    const auto hvr = rsrc(seg + L.hv, set_bytes);
    const auto* mask_words = as_const(reinterpret_cast<const uint32_t*>(seg + L.mask));
    const auto* counts = as_const(reinterpret_cast<const uint32_t*>(seg + L.count));

    // ---- the wave's tiles
    // first token of the wave's tile i; T where it has none (every load reads zeros, every token is masked)
    auto tile_token = [&](int i) __attribute__((always_inline)) -> int {
      const int u = chunk0 + tg + TG * i;
      int t = u * TOK;
      if (picked) {
        const int b = __builtin_amdgcn_readlane(my_block, i & 63);
        t = b < 0 ? T : b * kBlockTokens + (u % S::TPB) * TOK;
      }
      return i < n && u < end ? t : T;
    };

    // ---- loads
    // K in the operand's layout: lane (lc, lg) holds pieces 4 kk + lg of its token(s)
    auto load_k = [&](int t0, uint32_t lane_off, uint4 (&x)[NLD]) __attribute__((always_inline)) {
      const uint32_t base = t0 < T ? (uint32_t)t0 * (C8 ? D : RB) : kOob;
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        uint32_t step;
        if constexpr (C8 || F32)
          step = (uint32_t)i * 64;                                          // the next pieces of the row(s)
        else
          step = (uint32_t)(i / KK) * (quad_row<D, TY>(0, 1) * RB) + (uint32_t)(i % KK) * 64;
        x[i] = ld128<0>(kr, base + lane_off + step);
      }
    };
    // A tile row by row on its way to LDS: the wave's share of its loads
    constexpr int VLD = NLD > CG ? NLD / CG : 1;
    const bool v_live = cg * VLD < NLD;
    auto load_rowwise = [&](const __amdgpu_buffer_rsrc_t& r, int t0, uint4 (&x)[VLD]) __attribute__((always_inline)) {
      const uint32_t base = t0 < T && v_live ? (uint32_t)t0 * (C8 ? D : RB) : kOob;
#pragma unroll
      for (int i = 0; i < VLD; ++i) x[i] = ld128<0>(r, base + (uint32_t)lane * 16 + (uint32_t)(cg * VLD + i) * 1024);
    };
    // ... and into LDS (a padding row of an E4M3 block may hold anything: it goes in as zero)
    auto stage = [&](uint8_t* tile, const uint4 (&v)[VLD], int t0) __attribute__((always_inline)) {
      if (CG > 1 && !v_live) return;
#pragma unroll
      for (int j = 0; j < VLD; ++j) {
        const int i = cg * VLD + j;
        if constexpr (C8) {
          constexpr int half = kC8Block / D / 2;
          const int row = i * 2 * half + lane / (D / 8), pc = lane % (D / 8);
          uint4 x = widen8(v[j].x, v[j].y), y = widen8(v[j].z, v[j].w);
          if (t0 + TOK > T) {
            if (t0 + row >= T) x = make_uint4(0, 0, 0, 0);
            if (t0 + row + half >= T) y = make_uint4(0, 0, 0, 0);
          }
          *reinterpret_cast<uint4*>(tile + piece_at<D, TY>(row, pc)) = x;
          *reinterpret_cast<uint4*>(tile + piece_at<D, TY>(row + half, pc)) = y;
        } else {
          *reinterpret_cast<uint4*>(tile + piece_at<D, TY>(i * RPL + lane / NP, lane % NP)) = v[j];
        }
      }
    };
    uint32_t k_off;
    if constexpr (C8) {
      constexpr int half = kC8Block / D / 2;
      k_off = (uint32_t)(kC8Block * (lc / half) + 16 * ((lc % half) * (D / 8) + lg));
    } else {
      k_off = (uint32_t)((quad_row<D, TY>(lc >> 2, 0) + (lc & 3)) * RB + lg * 16);
    }

    auto load_entries = [&](const __amdgpu_buffer_rsrc_t& ir, const __amdgpu_buffer_rsrc_t& xr, int t0, int chunk, Entries& e) __attribute__((always_inline)) {
      const uint32_t e0 = (uint32_t)t0 * k + 8u * (uint32_t)chunk;
      const bool ok = t0 < T && chunk < TOK / 8 * k;
      const uint32_t vo = ok ? e0 * C : kOob;
      if constexpr (C == 1) {
        const uint2 a = ld64(xr, vo);
        e.v0 = make_uint4(a.x, a.y, 0, 0);
      } else {
        e.v0 = ld128<0>(xr, vo);
        if constexpr (C == 4) e.v1 = ld128<0>(xr, vo + 16);
      }
      if constexpr (q4) {
        const uint32_t io = ok ? e0 * 2 : kOob;
        e.ix = ld128<0>(ir, io);
        e.prev = (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(ir, ok && e0 > 0 ? io - 2 : kOob, 0, 0);
        e.nix = __builtin_amdgcn_raw_buffer_load_b32(ir, io + 16, 0, 0);
        if constexpr (C == 1) {
          e.nv0 = (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(xr, vo + 8, 0, 0);
        } else if constexpr (C == 2) {
          e.nv0 = __builtin_amdgcn_raw_buffer_load_b32(xr, vo + 16, 0, 0);
        } else {
          const uint2 a = ld64(xr, vo + 32);
          e.nv0 = a.x;
          e.nv1 = a.y;
        }
      } else {
        const uint2 a = ld64(ir, ok ? e0 : kOob);
        e.ix = make_uint4(a.x, a.y, 0, 0);
      }
    };
    // entry i of the chunk as fp32 (8 and 9: the two after it)
    auto value = [&](const Entries& e, int i) __attribute__((always_inline)) -> float {
      if constexpr (C == 4) {
        return as_f32(i < 4 ? word(e.v0, i) : i < 8 ? word(e.v1, i - 4) : i == 8 ? e.nv0 : e.nv1);
      } else if constexpr (C == 2) {
        const uint32_t w = i < 8 ? word(e.v0, i / 2) : e.nv0;
        return (i & 1) ? bf16_hi(w) : bf16_lo(w);
      } else {
        const uint32_t raw = i < 8 ? word(e.v0, i / 4) : e.nv0;
        const uint32_t w = (i & 2) && i < 8 ? e4m3x2_bf16<true>(raw) : e4m3x2_bf16<false>(raw);
        return (i & 1) ? bf16_hi(w) : bf16_lo(w);
      }
    };
    auto code = [&](const Entries& e, int i) __attribute__((always_inline)) -> uint32_t {  // blocks of four
      const uint32_t w = i < 8 ? word(e.ix, i / 2) : e.nix;
      return (i & 1) ? w >> 16 : w & 0xFFFFu;
    };
    // Where the chunk's entries go in R and what goes there.  No branch: an entry that has no place (of a token
    // behind the last, of a chunk behind the tile, or summed into its channel's first) goes to the row behind R, so
    // that the products of the rest of the tile can fill the waits.
    struct Placed {
      uint32_t at[8];
      float x[8];       // blocks of four, fp32
      uint32_t w[4];    // pairs in bf16: the stored values with the layer's sign, two a word
    };
    auto place = [&](const Entries& e, int chunk, int held, Placed& p) __attribute__((always_inline)) {  // held: tokens of the tile
      const bool live = chunk < TOK / 8 * k;
      const int e0 = 8 * chunk;
      int t = (int)by_topk.div((uint32_t)e0), j = e0 - t * k;  // token of the tile, entry of the token
      uint32_t base[8], perm[8];  // of an entry's row: its first byte, the permutation of its channels
      bool starts[10];            // the entry is its token's first
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (RES == kFewEntries && i > 0) {  // k is a multiple of eight: a chunk is of one token
          base[i] = base[0];
          perm[i] = perm[0];
          starts[i] = false;
          continue;
        }
        const int r = live && t < held ? t : TOK;
        base[i] = (uint32_t)(r * RB);
        perm[i] = (piece_at<D, TY>(r, 0) - base[i]) / S::E;
        starts[i] = j == 0;
        if constexpr (RES == kManyEntries) {
          const bool next = ++j == k;
          j = next ? 0 : j;
          t += next;
        }
      }
      if constexpr (RES == kFewEntries) {
        starts[8] = j + 8 == k;
        starts[9] = false;
      } else {
        starts[8] = j == 0;
        starts[9] = j + 1 == k || k == 1;
      }
      if constexpr (!q4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p.at[i] = base[i] + (((word(e.ix, i / 4) >> (8 * (i & 3))) & (D - 1)) ^ perm[i]) * S::E;
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < 8; ++i) p.x[i] = w1 * value(e, i);
        } else {
          const uint4 v = C8 ? widen8(e.v0.x, e.v0.y) : e.v0;
          const uint32_t sign = w1 < 0.f ? 0x80008000u : 0u;
#pragma unroll
          for (int i = 0; i < 4; ++i) p.w[i] = word(v, i) ^ sign;
        }
      } else {
        // a channel's up to three frequencies are neighbours (codes 4 c + j ascend): the first of them takes the sum
        float x[10];
        const float a = w1, b = w2, c = w3;
#pragma unroll
        for (int i = 0; i < 10; ++i) {
          const uint32_t f = code(e, i) & 3u;
          const float lo = f == 1u ? a : b;
          x[i] = (f == 3u ? c : lo) * value(e, i);
        }
#pragma unroll
        for (int i = 8; i >= 0; --i) x[i] += !starts[i + 1] && (code(e, i + 1) ^ code(e, i)) < 4u ? x[i + 1] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool first = starts[i] || ((i ? code(e, i - 1) : e.prev) ^ code(e, i)) >= 4u;
          p.at[i] = (first ? base[i] : (uint32_t)(TOK * RB)) + (((code(e, i) >> 2) & (D - 1)) ^ perm[i]) * S::E;
          p.x[i] = x[i];
        }
      }
    };
    // rest: what the bf16 rounding of the values leaves
    auto store = [&](uint8_t* rt, const Placed& p, bool rest) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (F32) {
          *reinterpret_cast<float*>(rt + p.at[i]) = p.x[i];
        } else if constexpr (!q4) {
          *reinterpret_cast<uint16_t*>(rt + p.at[i]) = (uint16_t)((i & 1) ? p.w[i / 2] >> 16 : p.w[i / 2]);
        } else {
          const uint32_t hi = f32_to_bf16_bits(p.x[i]);
          *reinterpret_cast<uint16_t*>(rt + p.at[i]) = (uint16_t)(rest ? f32_to_bf16_bits(rest_of(p.x[i], bf16_to_f32((uint16_t)hi))) : hi);
        }
      }
    };
    Placed placed[NCH];
    auto place_all = [&](const Entries (&e)[NCH], int t0) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) place(e[i], lane + 64 * i, T - t0, placed[i]);
    };
    auto scatter = [&](uint8_t* rt, const __amdgpu_buffer_rsrc_t& ir, const __amdgpu_buffer_rsrc_t& xr, int t0, bool rest) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) store(rt, placed[i], rest);
      if constexpr (RES == kManyEntries) {
        for (int c = lane + 64 * NCH; c < TOK / 8 * k; c += 64) {
          Entries f;
          load_entries(ir, xr, t0, c, f);
          Placed p;
          place(f, c, T - t0, p);
          store(rt, p, rest);
        }
      }
    };

    // token-level set: the tile's part of the mask, and the set tokens before it
    auto load_mask = [&](int t0, uint32_t& mw, uint32_t& rank) __attribute__((always_inline)) {
      const int t = min(t0, T - 1), w = t >> 5;  // (one read of the chunk's four words: a mask plane is padded)
      const auto* quad = mask_words + (w & ~3);
      const uint32_t m0 = quad[0], m1 = quad[1], m2 = quad[2], m3 = quad[3], before = counts[t >> 7];
      const int i = w & 3;
      mw = i == 0 ? m0 : i == 1 ? m1 : i == 2 ? m2 : m3;
      rank = before + (i > 0 ? __builtin_popcount(m0) : 0) + (i > 1 ? __builtin_popcount(m1) : 0) + (i > 2 ? __builtin_popcount(m2) : 0);
      if constexpr (TOK == 16) {
        rank += t & 16 ? __builtin_popcount(mw & 0xFFFFu) : 0;
        mw = t & 16 ? mw >> 16 : mw & 0xFFFFu;
      }
      const int held = T - t0;
      mw = held <= 0 ? 0u : held < TOK ? mw & ((1u << held) - 1u) : mw;
    };
    constexpr int HB = 16 / S::E * C;  // stored bytes of a 16-byte LDS piece
    struct SetRows {
      uint4 x[q4 ? 3 : 1];
    };
    // rows `from` .. of the tile's set tokens, RPL of them: the lane's piece
    auto load_rows = [&](const __amdgpu_buffer_rsrc_t& r, uint32_t mw, uint32_t rank, int from, SetRows& x) __attribute__((always_inline)) {
      const uint32_t row = rank + (uint32_t)(from + lane / NP);
      const bool ok = from + lane / NP < __builtin_popcount(mw);
#pragma unroll
      for (int f = 0; f < (q4 ? 3 : 1); ++f) {
        const uint32_t off = ok ? (row * (q4 ? 3u : 1u) + f) * (uint32_t)(D * C) + (uint32_t)(lane % NP) * HB : kOob;
        if constexpr (HB == 8) {
          const uint2 a = ld64(r, off);
          x.x[f] = make_uint4(a.x, a.y, 0, 0);
        } else {
          x.x[f] = ld128<0>(r, off);
        }
      }
    };
    // The rows into R: the lane's is that of the (lane / NP)-th set bit of `left`, which loses RPL bits.  A lane past
    // the set writes to the row behind R.
    auto put_rows = [&](uint8_t* rt, const SetRows& x, uint32_t& left, bool rest) __attribute__((always_inline)) {
      int t = TOK;
#pragma unroll
      for (int i = 0; i < RPL; ++i) {
        const int ti = left ? __builtin_ctz(left) : TOK;
        t = lane / NP == i ? ti : t;
        left &= left - 1;
      }
      uint32_t ow[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
          float y = w1 * as_f32(word(x.x[0], i));
          if constexpr (q4) y = fmaf(w3, as_f32(word(x.x[2], i)), fmaf(w2, as_f32(word(x.x[1], i)), y));
          ow[i] = as_u32(y);
        } else {
          auto pair = [&](const uint4& v) __attribute__((always_inline)) -> uint32_t {
            if constexpr (C8) return (i & 1) ? e4m3x2_bf16<true>(word(v, i / 2)) : e4m3x2_bf16<false>(word(v, i / 2));
            return word(v, i);
          };
          const uint32_t a = pair(x.x[0]);
          if constexpr (q4) {
            const uint32_t bb = pair(x.x[1]), cc = pair(x.x[2]);
            const float y0 = fmaf(w3, bf16_lo(cc), fmaf(w2, bf16_lo(bb), w1 * bf16_lo(a)));
            const float y1 = fmaf(w3, bf16_hi(cc), fmaf(w2, bf16_hi(bb), w1 * bf16_hi(a)));
            const uint32_t hi = cvt_bf16x2(y0, y1);
            ow[i] = rest ? cvt_bf16x2(rest_of(y0, bf16_lo(hi)), rest_of(y1, bf16_hi(hi))) : hi;
          } else {
            ow[i] = a ^ (w1 < 0.f ? 0x80008000u : 0u);
          }
        }
      }
      *reinterpret_cast<uint4*>(rt + piece_at<D, TY>(t, lane % NP)) = make_uint4(ow[0], ow[1], ow[2], ow[3]);
    };
    auto set_rows = [&](uint8_t* rt, const __amdgpu_buffer_rsrc_t& r, const SetRows& x, uint32_t mw, uint32_t rank, bool rest) __attribute__((always_inline)) {
      uint32_t left = mw;
      put_rows(rt, x, left, rest);
      for (int from = RPL; left; from += RPL) {  // more rows than travel ahead: loaded where they are used
        SetRows y;
        load_rows(r, mw, rank, from, y);
        put_rows(rt, y, left, rest);
      }
    };
    auto clear_r = [&](uint8_t* rt) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) *reinterpret_cast<uint4*>(rt + i * 1024 + lane * 16) = make_uint4(0, 0, 0, 0);
    };

    // ---- products
    f32x4_t s[NQ][TI];
    auto qk_piece = [&](const uint4& a, const uint4& b, int q, int i) __attribute__((always_inline)) {
      if constexpr (F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          s[q][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(as_f32(word(a, j)), as_f32(word(b, j)), s[q][i], 0, 0, 0);
      } else {
        s[q][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                          s[q][i], 0, 0, 0);
      }
    };
    // piece(i, kk): the A operand of 16 tokens and the kk-th channels
    auto qk = [&](auto piece) __attribute__((always_inline)) {
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        uint4 a[TI];
#pragma unroll
        for (int i = 0; i < TI; ++i) a[i] = piece(i, kk);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const uint4 b = qf[q][kk];
#pragma unroll
          for (int i = 0; i < TI; ++i) qk_piece(a[i], b, q, i);
        }
      }
    };
    // Operands in an LDS tile.  Pieces are permuted by XOR, and a tile starts at a multiple of a row, so the piece of
    // the kk-th channels (the c-th output tile) is the first one's address with some bits flipped.  (The addresses are
    // formed where they are used: held for all of a tile's reads they would take the registers that its loads need.)
    auto qk_tile = [&](const uint8_t* tile) __attribute__((always_inline)) {
      lds_fence();
      uint32_t at = (uint32_t)(tile - lds) + piece_at<D, TY>(quad_row<D, TY>(lc >> 2, 0) + (lc & 3), lg);
      asm("" : "+v"(at));
      qk([&](int i, int kk) __attribute__((always_inline)) -> uint4 {
        return *reinterpret_cast<const uint4*>(lds + (at ^ (uint32_t)(kk << 6)) + i * (quad_row<D, TY>(0, 1) * RB));
      });
      lds_fence();
    };
    // probabilities of the lane's tokens: bf16 operand words, or fp32
    uint32_t pb[NQ][4];
    auto pv = [&](const uint8_t* tile) __attribute__((always_inline)) {
      lds_fence();
      const uint32_t off = (uint32_t)(tile - lds);
      if constexpr (F32) {
        uint32_t at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          at[i] = off + piece_at<D, TY>(4 * lg + i, lc >> 2) + (lc & 3) * 4;
          asm("" : "+v"(at[i]));
        }
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a = *reinterpret_cast<const float*>(lds + (at[i] ^ (uint32_t)(c << 6)));
#pragma unroll
            for (int q = 0; q < NQ; ++q)
              acc[q][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, as_f32(pb[q][i]), acc[q][c], 0, 0, 0);
          }
      } else {
        // rows quad .. quad + 3 of both operands, channels 16 c ..: lane i of a group names row i / 4, channels 4 (i % 4) ..
        uint32_t at = off + piece_at<D, TY>(quad_row<D, TY>(lg, 0) + (lc >> 2), (lc & 3) >> 1) + (lc & 1) * 8;
        asm("" : "+v"(at));
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          i16x4_t h[2];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_i16x4_t*)(lds + (at ^ (uint32_t)(c << 5)) + i * (quad_row<D, TY>(0, 1) * RB)));
          const i16x8_t a = {h[0][0], h[0][1], h[0][2], h[0][3], h[1][0], h[1][1], h[1][2], h[1][3]};
#pragma unroll
          for (int q = 0; q < NQ; ++q)
            acc[q][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, make_uint4(pb[q][0], pb[q][1], pb[q][2], pb[q][3])),
                acc[q][c], 0, 0, 0);
        }
      }
      lds_fence();
    };

    // ---- what travels ahead of a tile
    struct Ahead {
      uint4 kv[CG == 1 ? NLD : VLD], vv[VLD];
      Entries ek[NCH], ev[NCH];
      SetRows sk, sv;
      uint32_t mask, rank;
      int t0;
    };
    auto load_res = [&](Ahead& b) __attribute__((always_inline)) {
      if constexpr (ENT) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
          load_entries(ikr, xkr, b.t0, lane + 64 * i, b.ek[i]);
          if constexpr (CG == 1) load_entries(ivr, xvr, b.t0, lane + 64 * i, b.ev[i]);
        }
      }
      if constexpr (SET) {
        load_rows(hkr, b.mask, b.rank, 0, b.sk);
        if constexpr (CG == 1) load_rows(hvr, b.mask, b.rank, 0, b.sv);
      }
    };
    // Tile `it` from its buffer, which then takes tile it + DEPTH.
    auto step = [&](Ahead& b, int it) __attribute__((always_inline)) {
      const int t0 = b.t0, tn = tile_token(it + DEPTH);
      const uint32_t mask = b.mask, rank = b.rank;
      b.t0 = tn;
      if constexpr (SET) load_mask(tn, b.mask, b.rank);
      const bool has = ENT || (SET && mask != 0);
      const bool edge = t0 + TOK > T;  // tokens of the tile past the last one

      stage(vt, b.vv, t0);
      load_rowwise(vr, tn, b.vv);
      if constexpr (CG > 1) {
        stage(kt, b.kv, t0);
        load_rowwise(kr, tn, b.kv);
      }
      if constexpr (CG > 1 && RES != 0) {
        if (has && role < roles) {
          const bool rest = REST && role >= 2;
          if constexpr (ENT) {
            place_all(b.ek, t0);
            scatter(rt, ikr, xkr, t0, rest);
          }
          if constexpr (SET) set_rows(rt, hkr, b.sk, mask, rank, rest);
        }
        load_res(b);
      }

      SetRows sv;  // V's rows, for their rest

      // K
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int i = 0; i < TI; ++i) s[q][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if constexpr (CG > 1) {
        hand_over();
        qk_tile(kt);
        if (has) {
          qk_tile(r_k);
          if constexpr (REST) qk_tile(r_rest);
        }
      } else {
        qk([&](int i, int kk) __attribute__((always_inline)) -> uint4 {
          if constexpr (C8)
            return i ? widen8(b.kv[kk].z, b.kv[kk].w) : widen8(b.kv[kk].x, b.kv[kk].y);
          else
            return b.kv[i * KK + kk];
        });
        load_k(tn, k_off, b.kv);
        if (has) {
          if constexpr (ENT) {
            place_all(b.ek, t0);
            scatter(rt, ikr, xkr, t0, false);
          }
          if constexpr (SET) set_rows(rt, hkr, b.sk, mask, rank, false);
          qk_tile(rt);
          if constexpr (REST) {
            if constexpr (ENT) scatter(rt, ikr, xkr, t0, true);
            if constexpr (SET) set_rows(rt, hkr, b.sk, mask, rank, true);
            qk_tile(rt);
          }
          clear_r(rt);
          lds_fence();
          if constexpr (ENT) {
            place_all(b.ev, t0);
            scatter(rt, ivr, xvr, t0, false);
          }
          if constexpr (SET) set_rows(rt, hvr, b.sv, mask, rank, false);
        }
        if constexpr (SET && REST) sv = b.sv;
        load_res(b);
      }

      // softmax
      if (edge) {
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (t0 + quad_row<D, TY>(lg, i) + r >= T) s[q][i][r] = -INFINITY;
      }
      float mx[NQ];
      bool move = false;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        mx[q] = s[q][0][0];
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) mx[q] = fmaxf(mx[q], s[q][i][r]);
        mx[q] = scale * col_max(mx[q]);
        move = move || mx[q] > m[q] + kSlack;
      }
      if (__any(move)) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const float mn = fmaxf(m[q], mx[q]);
          const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[q] - mn);
          m[q] = mn;
          l[q] *= f;
#pragma unroll
          for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[q][c][r] *= f;
        }
      }
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float ref = m[q] == -INFINITY ? 0.f : m[q];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < TI; ++i) {
          float p[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            p[r] = __builtin_amdgcn_exp2f(fmaf(s[q][i][r], scale, -ref));
            sum += p[r];
          }
          if constexpr (F32) {
#pragma unroll
            for (int r = 0; r < 4; ++r) pb[q][r] = as_u32(p[r]);
          } else {
            pb[q][2 * i] = cvt_bf16x2(p[0], p[1]);
            pb[q][2 * i + 1] = cvt_bf16x2(p[2], p[3]);
          }
        }
        l[q] += sum;
      }

      // V
      pv(vt);
      if (has) {
        pv(r_v);
        if constexpr (REST) {
          if constexpr (CG == 1) {
            if constexpr (ENT) scatter(rt, ivr, xvr, t0, true);
            if constexpr (SET) set_rows(rt, hvr, sv, mask, rank, true);
          }
          pv(r_vrest);
        }
      }
      if constexpr (CG > 1) hand_over();
      if (has && role < roles) {
        clear_r(rt);
        lds_fence();
      }
    };

    if constexpr (RES != 0) {
      if (role < roles) clear_r(rt);
    }
    Ahead ahead[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      Ahead& b = ahead[d];
      b.t0 = tile_token(d);
      b.mask = b.rank = 0;
      if constexpr (SET) load_mask(b.t0, b.mask, b.rank);
      load_rowwise(vr, b.t0, b.vv);
      if constexpr (CG == 1)
        load_k(b.t0, k_off, b.kv);
      else
        load_rowwise(kr, b.t0, b.kv);
      load_res(b);
    }
    settle_queries();
#pragma unroll 1
    for (int it = 0; it < n; it += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        if (d > 0 && it + d >= n) break;
        step(ahead[d], it + d);
      }
    }
  };

  using std::integral_constant;
  using no = integral_constant<bool, false>;
  using yes = integral_constant<bool, true>;
  const bool res = mode == kResidual && (KIND == kTokenSet || k > 0);
  if (chunk0 < end && !bad_unit) {  // (the whole workgroup: the walk may have barriers)
    if constexpr (TY == kTyC8) {
      if (mode == kExact)
        walk(no{}, no{});
      else if (res)
        walk(yes{}, yes{});
      else
        walk(yes{}, no{});
    } else {
      if (res)
        walk(no{}, yes{});
      else
        walk(no{}, no{});
    }
  }

  if (res_cost && slot == slot0 && row0 == 0 && threadIdx.x == 0) P.shared_counts[head] = head_slots;

  // ---- the waves' records of a column tile meet in LDS, one tile after the other
  float* mg = reinterpret_cast<float*>(lds);  // [wave][column][MP]
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    if (row0 + 16 * q >= rows) break;
    __syncthreads();
    const float ls = col_sum(l[q]);
    if (lg == 0) {
      ml_lds[wave][lc][0] = m[q];
      ml_lds[wave][lc][1] = ls;
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
      *reinterpret_cast<f32x4_t*>(mg + (wave * 16 + lc) * MP + 16 * c + 4 * lg) = acc[q][c];
    __syncthreads();
    constexpr int TPC = 16 / CG;  // threads of a column
    const int col = threadIdx.x / TPC, sub = threadIdx.x % TPC, gr = col / 16, cl = col % 16;
    int sq, g;
    if (row_of(16 * (gr * NQ + q) + cl, sq, g)) {
      float M = -INFINITY;
#pragma unroll
      for (int t = 0; t < TG; ++t) M = fmaxf(M, ml_lds[t * CG + gr][cl][0]);
      float wt[TG], lt = 0.f;
#pragma unroll
      for (int t = 0; t < TG; ++t) {
        wt[t] = merge_weight(ml_lds[t * CG + gr][cl][0], M);
        lt = fmaf(wt[t], ml_lds[t * CG + gr][cl][1], lt);
      }
      float* rec = ws + ((((uint64_t)sq * hkv + head) * n_slots_total + slot) * G + g) * RS;
#pragma unroll
      for (int c = 0; c < D / (4 * TPC); ++c) {
        const int ch = 4 * (TPC * c + sub);
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < TG; ++t) o += wt[t] * *reinterpret_cast<const f32x4_t*>(mg + ((t * CG + gr) * 16 + cl) * MP + ch);
        if (bad_unit) o = f32x4_t{NAN, NAN, NAN, NAN};
        *reinterpret_cast<f32x4_t*>(rec + ch) = o;
      }
      if (sub == 0) {
        rec[D] = bad_unit ? 0.f : M;
        rec[D + 1] = bad_unit ? 1.f : lt;
      }
    }
  }
}

// NQ, CG: of the shared parts' workgroups; those of single sequences have one column tile and four token groups.  (The
// two kinds in one launch: the second fills the CUs that the first leaves one by one.)
template <int D, int NQ, int CG, int TY, int KIND, bool q4>
__global__ __launch_bounds__(256, parts_per_cu(KIND, q4)) void parts_kernel(PartsParams P) {
  constexpr int own = PartsLds<D, 1, TY, q4>::BYTES, both = PartsLds<D, CG, TY, q4>::BYTES;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[own > both ? own : both];
  __shared__ float ml_lds[4][16][2];
  const bool shared = blockIdx.x < P.shared_wgs;
  if constexpr (CG * NQ > 1) {
    if (shared) {
      parts_body<D, NQ, CG, TY, KIND, q4>(P, P.side[1], blockIdx.x, lds, ml_lds);
      return;
    }
  }
  parts_body<D, 1, 1, TY, KIND, q4>(P, P.side[shared ? 1 : 0], shared ? blockIdx.x : blockIdx.x - P.shared_wgs, lds, ml_lds);
}

template <int D, int TY, int KIND, bool q4>
static hipError_t launch_parts_kind(const PartsParams& P, hipStream_t s) {
  const dim3 grid(P.shared_wgs + (uint32_t)P.hkv * (uint32_t)P.side[0].n_slots * (uint32_t)P.batch), block(256);
  if (P.cols == 16) {
    hipLaunchKernelGGL((parts_kernel<D, 1, 1, TY, KIND, q4>), grid, block, 0, s, P);
  } else if (P.cols == 128) {
    hipLaunchKernelGGL((parts_kernel<D, 2, 4, TY, KIND, q4>), grid, block, 0, s, P);
  } else if (P.cols == 32) {  // (where parts_cols has it)
    if constexpr (TY != parts::kTyF32 && KIND != kManyEntries)
      hipLaunchKernelGGL((parts_kernel<D, 2, 1, TY, KIND, q4>), grid, block, 0, s, P);
    else
      return hipErrorInvalidValue;
  } else {
    if constexpr (TY != parts::kTyF32 && (KIND == kManyEntries || (TY == parts::kTyBf16 && !q4)))
      hipLaunchKernelGGL((parts_kernel<D, 1, 4, TY, KIND, q4>), grid, block, 0, s, P);
    else
      return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <int D, int TY>
static hipError_t launch_parts_ty(const PartsParams& P, hipStream_t s) {
  const bool quad = P.bsize == 4;
  if (P.tokres)
    return quad ? launch_parts_kind<D, TY, kTokenSet, true>(P, s) : launch_parts_kind<D, TY, kTokenSet, false>(P, s);
  if (P.topk % 8 == 0 && parts::TileOf<D, TY>::TOK / 8 * P.topk <= 64)
    return quad ? launch_parts_kind<D, TY, kFewEntries, true>(P, s) : launch_parts_kind<D, TY, kFewEntries, false>(P, s);
  return quad ? launch_parts_kind<D, TY, kManyEntries, true>(P, s) : launch_parts_kind<D, TY, kManyEntries, false>(P, s);
}

}  // namespace fdkv
