// Causal attention of packed prompts (fdkv_prompt_attn):
//   o_i = sum_j softmax_j(q_i . k_j scale) v_j,  j <= K - N + i,
// for the N query tokens i of a sequence and its K keys (the last N of which
// are the query tokens' own).
//
// A workgroup takes 128 query rows (token, head of the group) of one sequence
// and KV head, so that a group's heads share every key tile; its four waves
// take 32 rows each and walk tiles of 64 or 32 keys that they stage
// together in LDS, the next tile's loads in flight behind the current one:
//   S^T = K Q^T    A: 32 keys x 16 channels from LDS, B: the queries, in registers;
//   softmax        a row lives on lanes l and l + 32; running max (moved only by more
//                  than 2^8) and sum in fp32;
//   O^T += V^T P^T the probabilities are the B operand where they lie (the keys of
//                  a lane's S^T registers are the keys of its B slots), A: transposed
//                  reads of the V tile.
// Tiles of query rows are taken from the call's last on down (of one prompt: those
// with more keys first), but for calls whose workgroups all run at once (`launch`).
// Workgroups of a KV head are hkv apart, which for eight heads keeps a head's keys in one XCD's L2.
// Probabilities are rounded to bf16 (2^-8 each at most) for the product, their sum is not.
// Calls of few rows and many keys split the keys over workgroups, whose
// (acc, m, l) records a second launch joins.
//
// What bounds it.  Long prompts: the card's power.  32768 tokens of 32 + 8 heads of 128
// (bf16) take 7.5 ms, 1.18 PFLOP/s, where a large matrix product of the library's reaches 1.43, at some 1.7 GHz
// with the matrix units busy 60% of the time; with inputs of zeros the same call takes 4.99 ms, 1.76 PFLOP/s, and the
// library's product reaches 1.81.  Key tiles that pass through registers on their way to LDS spill (2028 us for 8191
// tokens, now 496); 64 rows a wave, which halve what is read from LDS, leave one wave a SIMD (32768 tokens 8.8 ms), two
// groups of waves that take turns at the matrix units wait for their operands (8.7), the next tile's logits ahead of
// this one's softmax gain 1% where they have the registers, and three or four tiles in LDS instead of two gain nothing
// (32768 tokens 7.78 to 8.23 for 7.81, 2048 tokens 57 to 66 us for 51).  Prompts of 2048 tokens (51 us, 670 TFLOP/s) wait for their
// longest workgroups, a step of which takes 1.2 us without others beside it.  fp32: the matrix units (8192 tokens 140
// TFLOP/s of 154).
#include <algorithm>

#include "parts.h"
#include "rows_kernels.h"

namespace fdkv {

namespace {

using namespace parts;

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) uint8_t lds_u8_t;

template <int D, bool F32, int KEYS>
struct Prompt {
  static constexpr int E = F32 ? 4 : 2, RB = D * E, NP = RB / 16;
  static constexpr int KB = KEYS / 32;                // blocks of 32 keys
  static constexpr int TILE_BYTES = KEYS * RB;
  static constexpr int NL = TILE_BYTES / 4096;        // 16-byte loads of a thread, of K or V
  static constexpr int RPI = 64 / NP;                 // rows of a wave's load
  static constexpr int KS = F32 ? D / 8 : D / 16;     // operand pieces of a row, of a lane
  static constexpr int CB = D / 32;                   // blocks of 32 channels
  // Byte of a 16-byte piece of a row of a K tile: eight rows of one piece in distinct banks.
  static __device__ __forceinline__ uint32_t k_at(int row, int piece) {
    return (uint32_t)(row * RB + ((piece ^ k_flip(row)) << 4));
  }
  static __device__ __forceinline__ int k_flip(int row) { return row & (!F32 && D == 128 ? 15 : 7); }
  // ... of a V tile: a transposed read takes 64 bytes of four rows at once.  (fp32: 128 bytes of one.)
  static __device__ __forceinline__ uint32_t v_at(int row, int piece) {
    return (uint32_t)(row * RB + ((piece ^ v_flip(row)) << 4));
  }
  static __device__ __forceinline__ int v_flip(int row) { return F32 ? 0 : D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; }
};

// 16 bytes a lane from r + voff (+ i step) to LDS, lane l's at `to` (+ 4096 i) + 16 l.  The compiler does not see the
// loads: its own waits would hold up every LDS read until the loads in flight to the other half of the buffer have
// landed.  Nor does it see what has to lie between: five wait states from a vector instruction's write of a scalar
// register to its use as an address, one from the write of m0 to a load to LDS.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
// (m0 is the compiler's own register: it warns that what it holds is lost, which is what the clobber is to tell it)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds(u32x4_t r, uint32_t voff, uint32_t to) {
  asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(voff), "s"(r) : "memory", "m0");
}
template <int NL>
__device__ __forceinline__ void load_lds(u32x4_t r, uint32_t voff, uint32_t step, uint32_t to) {
  static_assert(NL == 2 || NL == 4, "loads of a tile");
  if constexpr (NL == 2)
    asm volatile(
        "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds" ::"s"(to),
        "s"(to + 4096), "v"(voff), "s"(r), "s"(__builtin_amdgcn_readfirstlane(step))
        : "memory", "m0");
  else
    asm volatile(
        "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen lds\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, %6 offen lds\n\t"
        "s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, %7 offen lds\n\t"
        "s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, %8 offen lds" ::"s"(to),
        "s"(to + 4096), "s"(to + 8192), "s"(to + 12288), "v"(voff), "s"(r), "s"(__builtin_amdgcn_readfirstlane(step)),
        "s"(__builtin_amdgcn_readfirstlane(2 * step)), "s"(__builtin_amdgcn_readfirstlane(3 * step))
        : "memory", "m0");
}
#pragma clang diagnostic pop
// A buffer of rows from `base` on (the callers stay within their rows).
__device__ __forceinline__ u32x4_t buffer_at(const uint8_t* base) {
  const uint64_t a = (uint64_t)(uintptr_t)base;
  return u32x4_t{(uint32_t)a, (uint32_t)(a >> 32) & 0xFFFFu, ~0u, 0x00020000u};
}

__device__ __forceinline__ float pair_max(float x) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Bits of a word of value rows that are set where a value in it is not finite.
template <bool F32>
__device__ __forceinline__ uint32_t odd_bits(uint32_t x) {
  return F32 ? ((x & 0x7F800000u) + 0x00800000u) & 0x80000000u : ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}
// The word with 0 in the place of such values.
template <bool F32>
__device__ __forceinline__ uint32_t without_odd(uint32_t x) {
  const uint32_t o = odd_bits<F32>(x);
  return F32 ? (o ? 0u : x) : x & ~((o >> 15) * 0xFFFFu);
}

// KEYS of a tile, workgroups to a CU.  (bf16 of 128 channels: tiles of 64 keys for calls of few workgroups, 32 for those of
// many, of which a CU then holds three.  us, tiles of 64 and 32: a prompt of 1000 tokens 26.7 and 28.9, 2048 tokens 53.5 and
// 57.3, 8191 tokens 515 and 512, 24 prompts of up to 2000 tokens 360 and 341, 32768 tokens 7770 and 7600, 250 tokens on 33018
// keys 288 and 295.)  64 channels: four workgroups, although bf16 then spills some registers outside of the loops (us, four
// and three, bf16: 2048 tokens 37.2 and 36.5, 8192 tokens 311 and 318, 32768 tokens 4651 and 4744, 24 prompts of up to 2000
// tokens 218 and 221; fp32: 1000 tokens 63.1 and 63.4, 8192 tokens 2006 and 2064, the 24 prompts 1275 and 1264).
constexpr int keys_of(int D, bool F32, bool many) { return F32 || (many && D == 128) ? 32 : 64; }
constexpr int per_cu(int D, bool F32, int keys) { return D == 64 ? 4 : F32 || keys == 64 ? 2 : 3; }
constexpr int kManyGroups = 1024, kCus = 256;

template <int D, bool F32, int KEYS>
__global__ __launch_bounds__(256, per_cu(D, F32, KEYS)) void prompt_attn_kernel(PromptParams P) {
  using S = Prompt<D, F32, KEYS>;
  constexpr int RB = S::RB, NP = S::NP, KB = S::KB, NL = S::NL, KS = S::KS, CB = S::CB, RS = D + 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[4 * S::TILE_BYTES];  // K, V; K, V of the next tile
  __shared__ __attribute__((aligned(16))) uint32_t odd_lds[2][4];          // by buffer and wave: V holds values that are not finite

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lr = lane & 31, lh = lane >> 5;
  const int g_shift = P.g_shift, G = 1 << g_shift;

  // ---- which rows: tile numbers count floor(G q_starts[s] / 128) + s from sequence s on
  const uint32_t y = P.by_hkv.div(blockIdx.x);
  const int head = (int)(blockIdx.x - y * P.hkv);
  const int split = P.splits > 1 ? (int)(y % (uint32_t)P.splits) : 0;
  const int turn = (int)(P.splits > 1 ? y / (uint32_t)P.splits : y);
  const int tile = turn < P.cut ? P.tiles - 1 - turn : turn - P.cut;
  // (lane i: the i-th of 64 sequences, everything about it in one trip to memory)
  int seq = -1, t0 = 0, t1 = 0, k0 = 0, K = 0;
  for (int s0 = 0; s0 < P.batch; s0 += 64) {
    const int s = min(s0 + lane, P.batch - 1);
    const int from = min(max(P.q_starts[s], 0), P.n_tokens), to = max(min(P.q_starts[s + 1], P.n_tokens), from);
    const int kf = P.k_starts ? min(max(P.k_starts[s], 0), P.rows) : 0;
    const int kn = min(max(P.k_lens[s], 0), P.rows - kf);
    const bool before = s0 + lane < P.batch && (int)(((int64_t)from << g_shift) / kPromptRows) + s <= tile;
    const int n = __builtin_popcountll(__ballot(before));  // (ascending starts: the first n lanes)
    if (n == 0) break;
    seq = s0 + n - 1;
    t0 = __builtin_amdgcn_readlane(from, n - 1);
    t1 = __builtin_amdgcn_readlane(to, n - 1);
    k0 = __builtin_amdgcn_readlane(kf, n - 1);
    K = __builtin_amdgcn_readlane(kn, n - 1);
    if (n < 64) break;
  }
  if (seq < 0) return;
  const int N = t1 - t0;
  const int64_t row0 = (int64_t)(tile - seq - (int)(((int64_t)t0 << g_shift) / kPromptRows)) * kPromptRows;
  const int64_t n_rows = (int64_t)N << g_shift;
  if (row0 < 0 || row0 >= n_rows) return;
  const int past = K - N;  // keys before the first query token's own (negative: the first tokens see none)

  const int64_t my_row = row0 + 32 * wave + lr;
  const bool live = my_row < n_rows;
  const int64_t row = live ? my_row : n_rows - 1;
  const int tok = t0 + (int)(row >> g_shift), g = (int)(row & (G - 1));
  const int lim = min(max(past + (int)(row >> g_shift) + 1, 0), K);  // keys that the row sees
  const int last_tok = (int)((min(row0 + kPromptRows, n_rows) - 1) >> g_shift);
  const int kmax = min(max(past + last_tok + 1, 0), K);              // ... that any row sees
  const int kmin = min(max(past + (int)(row0 >> g_shift) + 1, 0), K);  // ... that every row sees
  // ... that any row of the wave sees (0: it has no rows)
  const int64_t wrow = row0 + 32 * wave;
  const int wmax = wrow < n_rows ? min(max(past + (int)((min(wrow + 32, n_rows) - 1) >> g_shift) + 1, 0), K) : 0;
  int kb = 0, ke = kmax;
  if (P.splits > 1) {
    const int per = ((kmax + KEYS - 1) / KEYS + P.splits - 1) / P.splits * KEYS;
    kb = min(split * per, kmax);
    ke = min(kb + per, kmax);
  }

  // ---- queries
  uint4 qf[KS];
  {
    const uint8_t* src = static_cast<const uint8_t*>(P.q) + (int64_t)tok * P.q_stride + (int64_t)(head * G + g) * RB;
    const uint32_t keep = P.scale_log2 != 0.f ? 0xFFFFFFFFu : 0u;
    const uint32_t sign = P.scale_log2 < 0.f ? (F32 ? 0x80000000u : 0x80008000u) : 0u;  // the largest product is the largest logit
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const uint4 v = *reinterpret_cast<const uint4*>(src + 32 * j + 16 * lh);
      qf[j] = make_uint4((v.x ^ sign) & keep, (v.y ^ sign) & keep, (v.z ^ sign) & keep, (v.w ^ sign) & keep);
    }
  }
  const float scale = P.scale_log2 == 0.f ? 1.f : fabsf(P.scale_log2);

  float m = -INFINITY, l = 0.f;
  float ref = 0.f, top = -INFINITY;  // m, or 0 where there is none; the product that moves it
  f32x16_t acc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;

  const uint8_t* kbase = static_cast<const uint8_t*>(P.k) + seq * P.k_seq + head * P.k_head + k0 * P.k_row;
  const uint8_t* vbase = static_cast<const uint8_t*>(P.v) + seq * P.v_seq + head * P.v_head + k0 * P.v_row;
  // the thread's place in a wave's load: rows RPI apart from wave to wave, 4 RPI from load to load (the permutation of
  // the pieces has that period)
  constexpr int RPI = S::RPI;
  const int prow = RPI * wave + lane / NP, piece = lane % NP;
  const uint32_t kp = (uint32_t)((piece ^ S::k_flip(prow)) * 16), vp = (uint32_t)((piece ^ S::v_flip(prow)) * 16);
  const int k_row = (int)P.k_row, v_row = (int)P.v_row;
  const uint32_t k_off = prow * k_row + kp, v_off = prow * v_row + vp;
  const uint32_t to0 = (uint32_t)(uintptr_t)(lds_u8_t*)lds + wave * 1024;
  auto load = [&](int k, int b) __attribute__((always_inline)) {
    const int n = ke - k;
    const uint32_t to = to0 + b * 2 * S::TILE_BYTES;
    const auto kr = buffer_at(kbase + (int64_t)k * k_row), vr = buffer_at(vbase + (int64_t)k * v_row);
    if (n >= KEYS) {
      load_lds<NL>(kr, k_off, 4 * RPI * k_row, to);
      load_lds<NL>(vr, v_off, 4 * RPI * v_row, to + S::TILE_BYTES);
    } else {  // the last row stands in for those behind it, whose probabilities are 0
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = min(prow + 4 * RPI * i, n - 1);
        load_lds(kr, r * k_row + kp, to + 4096 * i);
        load_lds(vr, r * v_row + vp, to + S::TILE_BYTES + 4096 * i);
      }
    }
  };

  auto step = [&](const uint8_t* buf, int k, auto masked, auto blocks) __attribute__((always_inline)) {
    constexpr int KB = decltype(blocks)::value;  // blocks of 32 keys: the tile's first ones
    // Pieces are permuted by XOR and tiles start at multiples of a row, so an operand's address is the first one's with
    // some bits flipped.  (Formed where they are used: held for a whole tile they would take the operands' registers.)
    uint32_t ka = (uint32_t)(buf - lds) + S::k_at(lr, lh);
    uint32_t va = (uint32_t)(buf - lds) + S::TILE_BYTES +
                  (F32 ? S::v_at(4 * lh, 0) + lr * 4
                       : S::v_at(4 * lh + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + (lane & 1) * 8);
    asm("" : "+v"(ka), "+v"(va));
    f32x16_t s[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const uint4 op = *reinterpret_cast<const uint4*>(lds + (ka ^ (uint32_t)(j << 5)) + 32 * b * RB);
        if constexpr (F32) {
#pragma unroll
          for (int w = 0; w < 4; ++w)
            s[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(as_f32(word(op, w)), as_f32(word(qf[j], w)), s[b], 0, 0, 0);
        } else {
          s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, op), __builtin_bit_cast(bf16x8_t, qf[j]), s[b], 0, 0, 0);
        }
      }
      lds_fence();
    }
    if constexpr (decltype(masked)::value) {
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (k + 32 * b + 8 * (i / 4) + 4 * lh + i % 4 >= lim) s[b][i] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
    if (__any(mx > top)) {  // (of the lane's keys: the row's other lane looks at its own)
      const float mn = fmaxf(m, scale * pair_max(mx));
      const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      ref = mn == -INFINITY ? 0.f : mn;
      top = mn == -INFINITY ? -INFINITY : (mn + kSlack) / scale;
      l *= f;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] *= f;
    }
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], scale, -ref));
        l += s[b][i];
      }
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int c = 0; c < CB; ++c) {
            const float v = *reinterpret_cast<const float*>(lds + va + (8 * (i / 4) + i % 4) * RB + 128 * c);
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[b][i], acc[c], 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // keys 32 b + 16 h ..
          const uint4 pb = make_uint4(cvt_bf16x2(s[b][8 * h], s[b][8 * h + 1]), cvt_bf16x2(s[b][8 * h + 2], s[b][8 * h + 3]),
                                      cvt_bf16x2(s[b][8 * h + 4], s[b][8 * h + 5]), cvt_bf16x2(s[b][8 * h + 6], s[b][8 * h + 7]));
#pragma unroll
          for (int c = 0; c < CB; ++c) {
            i16x4_t x[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
              x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(lds + (va ^ (uint32_t)(c << 6)) + (32 * b + 16 * h + 8 * u) * RB));
            const i16x8_t av = {x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]};
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, av), __builtin_bit_cast(bf16x8_t, pb), acc[c], 0, 0, 0);
          }
          lds_fence();
        }
      }
    }
  };

#pragma unroll
  for (int j = 0; j < KS; ++j) asm volatile("" : "+v"(qf[j].x), "+v"(qf[j].y), "+v"(qf[j].z), "+v"(qf[j].w));  // (waited for here, not in the loop)
  if (kb < ke) load(kb, 0);
  int k = kb, b = 0;
  // A key that a row does not see has the probability 0, which takes its value out of the product where that is finite.  In
  // tiles that not every row sees all of, values that are not are set to 0, each by the thread that loaded it, and added
  // afterwards to the rows that see them.  (One look at a thread's pieces of a tile: 0.1 to 0.5 us of a call, 1000 tokens 25.8
  // and 26.3 us, 8191 tokens as long as without.)
  uint8_t* const mine_v = lds + S::TILE_BYTES + wave * 1024 + lane * 16;
  auto take_odd = [&]() __attribute__((always_inline)) {
    uint32_t o = 0;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const uint4 w = *reinterpret_cast<const uint4*>(mine_v + b * 2 * S::TILE_BYTES + 4096 * i);
      o |= odd_bits<F32>(w.x) | odd_bits<F32>(w.y) | odd_bits<F32>(w.z) | odd_bits<F32>(w.w);
    }
    const bool any = __any(o != 0);
    if (any) {
#pragma unroll 1
      for (int i = 0; i < NL; ++i) {
        uint4* at = reinterpret_cast<uint4*>(mine_v + b * 2 * S::TILE_BYTES + 4096 * i);
        const uint4 w = *at;
        *at = make_uint4(without_odd<F32>(w.x), without_odd<F32>(w.y), without_odd<F32>(w.z), without_odd<F32>(w.w));
      }
    }
    if (lane == 0) odd_lds[b][wave] = any;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  auto add_odd = [&]() __attribute__((always_inline)) {
    const int end = min(min(k + KEYS, ke), wmax);
#pragma unroll 1
    for (int key = k; key < end; ++key) {
      const uint8_t* src = vbase + (int64_t)key * v_row + 4 * lh * S::E;
      const uint32_t sees = key < lim ? ~0u : 0u;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint4 v;  // fp32
          if constexpr (F32) {
            v = *reinterpret_cast<const uint4*>(src + (32 * c + 8 * i) * 4);
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(src + (32 * c + 8 * i) * 2);
            v = make_uint4(x.x << 16, x.x & 0xFFFF0000u, x.y << 16, x.y & 0xFFFF0000u);
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint32_t w = word(v, u), keep = (uint32_t)((int32_t)odd_bits<true>(w) >> 31);
            acc[c][4 * i + u] += as_f32(w & keep & sees);
          }
          asm("" : "+v"(acc[c]));  // (one after another: it is rare, and its registers are the loop's)
        }
    }
  };
  auto next = [&](auto masked) __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if constexpr (decltype(masked)::value) take_odd();
    __builtin_amdgcn_s_barrier();
    lds_fence();
    if (k + KEYS < ke) load(k + KEYS, b ^ 1);
    const uint8_t* buf = lds + b * 2 * S::TILE_BYTES;
    if constexpr (!decltype(masked)::value)
      step(buf, k, masked, std::integral_constant<int, KB>{});
    else if (KB == 1 || k + 32 >= wmax) {
      if (k < wmax) step(buf, k, masked, std::integral_constant<int, 1>{});
    } else {
      step(buf, k, masked, std::integral_constant<int, KB>{});
    }
    if constexpr (decltype(masked)::value) {
      const uint4 o = *reinterpret_cast<const uint4*>(odd_lds[b]);
      if (__builtin_amdgcn_readfirstlane((int)(o.x | o.y | o.z | o.w))) add_odd();
    }
    k += KEYS;
    b ^= 1;
  };
  const int whole = min(ke, kmin / KEYS * KEYS);  // keys of tiles that every row sees all of (kb is a multiple of KEYS)
  while (k < whole) next(std::false_type{});
  while (k < ke) next(std::true_type{});
  l = pair_sum(l);
  if (P.splits > 1) {
    if (!live) return;
    float* rec = P.ws + (((int64_t)split * P.n_tokens + tok) * P.hq + head * G + g) * RS;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4_t*>(rec + 32 * c + 8 * i + 4 * lh) = f32x4_t{acc[c][4 * i], acc[c][4 * i + 1], acc[c][4 * i + 2], acc[c][4 * i + 3]};
    if (lh == 0) *reinterpret_cast<float2*>(rec + D) = make_float2(m, l);
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;  // 0: the row sees no key
  if constexpr (F32) {
    if (!live) return;
    float* out = static_cast<float*>(P.out) + ((int64_t)tok * P.hq + head * G + g) * D;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4_t*>(out + 32 * c + 8 * i + 4 * lh) =
            f32x4_t{acc[c][4 * i] * inv, acc[c][4 * i + 1] * inv, acc[c][4 * i + 2] * inv, acc[c][4 * i + 3] * inv};
  } else {
    // Through LDS, so that whole rows are written at once, 32 of a wave: in the half that no wave reads any more, or, where
    // that is too small, in all of it once every wave is done.
    constexpr bool HALF = 2 * S::TILE_BYTES >= 4 * 32 * RB;
    static_assert(4 * S::TILE_BYTES >= 4 * 32 * RB, "LDS for the rows of four waves");
    if constexpr (!HALF) __syncthreads();
    uint8_t* mine = lds + (HALF ? b * 2 * S::TILE_BYTES : 0) + wave * 32 * RB;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint2*>(mine + lr * RB + (((4 * c + i) ^ (lr & (NP - 1))) << 4) + 8 * lh) =
            make_uint2(cvt_bf16x2(acc[c][4 * i] * inv, acc[c][4 * i + 1] * inv), cvt_bf16x2(acc[c][4 * i + 2] * inv, acc[c][4 * i + 3] * inv));
    lds_fence();
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) {
      const int r = RPI * i + lane / NP;
      const int64_t at = row0 + 32 * wave + r;
      const uint4 w = *reinterpret_cast<const uint4*>(mine + r * RB + ((piece ^ (r & (NP - 1))) << 4));
      if (at < n_rows)
        *(reinterpret_cast<uint4*>(static_cast<uint16_t*>(P.out) + ((int64_t)(t0 + (int)(at >> g_shift)) * P.hq + head * G + (int)(at & (G - 1))) * D) + piece) = w;
    }
  }
}

// Joins the splits' records of a query row: D / 4 lanes fold one record after another (four in flight), or, of many
// splits (WIDE), the D / 4-lane groups of a workgroup take turns and meet in LDS.
template <int D, bool BF16, bool WIDE>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptParams P) {
  constexpr int RS = D + 4, LPR = D / 4, NG = 256 / LPR, STEP = WIDE ? NG : 1, U = 4;
  __shared__ float ml_lds[NG][2];
  __shared__ __attribute__((aligned(16))) float o_lds[NG][D];
  const int rg = threadIdx.x / LPR, c4 = threadIdx.x % LPR;
  const int64_t rows = (int64_t)P.n_tokens * P.hq, row = WIDE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * NG + rg;
  if (row >= rows) return;
  // tokens of no sequence have no records and keep their outputs
  const int tok = (int)(row / P.hq);
  if (tok < as_const(P.q_starts)[0] || tok >= as_const(P.q_starts)[P.batch]) return;
  const float* base = P.ws + row * RS;
  float M = -INFINITY, l = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  auto fold = [&](float mi, float li, const f32x4_t& a) __attribute__((always_inline)) {
    const float mn = fmaxf(M, mi), fo = merge_weight(M, mn), fw = merge_weight(mi, mn);
    M = mn;
    l = l * fo + li * fw;
    o = o * fo + a * fw;
  };
  for (int i0 = WIDE ? rg : 0; i0 < P.splits; i0 += STEP * U) {
    float2 ml[U];
    f32x4_t a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* r = base + (int64_t)min(i0 + STEP * u, P.splits - 1) * rows * RS;
      ml[u] = *reinterpret_cast<const float2*>(r + D);
      a[u] = *reinterpret_cast<const f32x4_t*>(r + 4 * c4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + STEP * u < P.splits) fold(ml[u].x, ml[u].y, a[u]);
  }
  if constexpr (WIDE) {
    if (c4 == 0) {
      ml_lds[rg][0] = M;
      ml_lds[rg][1] = l;
    }
    *reinterpret_cast<f32x4_t*>(&o_lds[rg][4 * c4]) = o;
    __syncthreads();
    if (rg) return;
#pragma unroll
    for (int i = 1; i < NG; ++i) fold(ml_lds[i][0], ml_lds[i][1], *reinterpret_cast<const f32x4_t*>(&o_lds[i][4 * c4]));
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if constexpr (BF16)
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out) + row * D + 4 * c4) = make_uint2(cvt_bf16x2(o[0] * inv, o[1] * inv), cvt_bf16x2(o[2] * inv, o[3] * inv));
  else
    *reinterpret_cast<f32x4_t*>(static_cast<float*>(P.out) + row * D + 4 * c4) = o * inv;
}

template <int D, bool F32>
hipError_t launch(PromptParams P, hipStream_t s) {
  P.by_hkv.set((uint32_t)P.hkv);
  P.tiles = (int)(((int64_t)P.n_tokens << P.g_shift) / kPromptRows) + P.batch;
  const dim3 grid((unsigned)((int64_t)P.tiles * P.hkv * P.splits));
  // Workgroups w and w + 256 share a CU where all of a call's run at once: the first 256 go from the longest on down, the
  // others from the shortest on up (us, 2048 tokens 52 and 50.5, in fp32 369 and 281, two prompts of 1000 tokens 34.5 and 29;
  // with more workgroups, which take the place of those that end, the longest go first: 2600 tokens 69 and 73).
  const bool at_once = ((int64_t)P.n_tokens << P.g_shift) / kPromptRows * P.hkv <= 2 * kCus;
  P.cut = P.splits == 1 && at_once ? std::max(kCus / P.hkv, 1) : P.tiles;
  constexpr int few = keys_of(D, F32, false), many = keys_of(D, F32, true);
  if (few == many || grid.x <= kManyGroups)
    hipLaunchKernelGGL((prompt_attn_kernel<D, F32, few>), grid, dim3(256), 0, s, P);
  else
    hipLaunchKernelGGL((prompt_attn_kernel<D, F32, many>), grid, dim3(256), 0, s, P);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || P.splits == 1) return e;
  const int64_t rows = (int64_t)P.n_tokens * P.hq;
  constexpr int rpw = 256 / (D / 4);
  if (P.splits > 8)
    hipLaunchKernelGGL((prompt_join_kernel<D, !F32, true>), dim3((unsigned)rows), dim3(256), 0, s, P);
  else
    hipLaunchKernelGGL((prompt_join_kernel<D, !F32, false>), dim3((unsigned)((rows + rpw - 1) / rpw)), dim3(256), 0, s, P);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attn(const PromptParams& P, hipStream_t s) {
  if (P.n_tokens == 0) return hipSuccess;
  if (P.d == 128) return P.bf16 ? launch<128, false>(P, s) : launch<128, true>(P, s);
  return P.bf16 ? launch<64, false>(P, s) : launch<64, true>(P, s);
}

}  // namespace fdkv
