// Parameter blocks and launchers of the serving step around the decode: rotated
// rows, the index of sparse decode, decode over parts (internal to libfdkv).
#pragma once

#include "fdkv_kernels.h"

namespace fdkv {

// the rows of a step, normed and rotated, on their way into the exact cache
constexpr int kRopeTokens = 2;      // tokens of a workgroup of a long call ...
constexpr int kRopeMany = 1024;     // ... one of at least this many tokens
struct RopeParams {
  DivU by_rows, by_pairs;      // division by hq + 2 hkv and rot / 2
  const void* q;               // [n_tokens][hq][d], q_stride bytes a token
  const void* k;               // [n_tokens][hkv][d]
  const void* v;
  int64_t q_stride, k_stride, v_stride;
  const void* q_norm;          // [d] or null
  const void* k_norm;
  const double* inv_freq;      // [rot / 2]
  const int32_t* pos;          // [n_axes][n_tokens]
  const int32_t* seqs;         // [n_tokens] or null (token i is sequence i)
  const int32_t* rows;         // [n_tokens]
  void* q_out;                 // [n_tokens][hq][d]
  void* k_out;                 // [batch][hkv][cap][d]
  void* v_out;
  float eps;
  int n_tokens, hq, hkv, d, rot, batch, cap;
  bool interleaved, bf16;
  uint8_t axis[64];            // axis of every pair
};

// sparse decode: bounds of the keys of a block of tokens, and the blocks that a step reads
constexpr int kBlockTokens = 64;
struct BoundsParams {
  const void* k[kMaxPtrLayers];   // [hkv][seq_len][d] each
  void* out[kMaxPtrLayers];       // [hkv][cap][2][d] each
  int n_layers, hkv, seq_len, cap, d;
  bool bf16;
};
constexpr int kScoreBlocks = 32;  // blocks of a scoring workgroup
struct SelectParams {
  const int32_t* seq_lens;     // [batch]
  const void* bounds;          // [batch][hkv][cap][2][d], cap = ceil(max_seq_len / 64)
  const void* q;               // [batch][hq][d]
  double* ws;                  // [batch][hkv][G][cap]
  int32_t* blocks;             // [batch][hkv][n_sel]
  int32_t* counts;             // [batch][hkv]
  int batch, hkv, hq, d, max_seq_len, cap, n_first, n_last, n_sel;
  bool bf16;
};

// decode over parts (parts.h): whole spans, selected blocks, shared spans, the exact tail
struct PartsPart {
  const int32_t* lens;         // [batch] ([1] of a shared part)
  const uint8_t* cache;        // null: the exact tail
  const uint8_t* modes;        // [batch][blocks][hkv], 4-byte aligned ([1][..][..] of a shared part); the tail: lens
  const uint64_t* seg_off;     // as modes
  const int32_t* blocks;       // [batch][hkv][n_sel] selected blocks; every token: lens
  const int32_t* counts;       // [batch][hkv]; every token: lens
  int n_sel, max_len;          // n_sel 0: every token
};

// The parts of single sequences, or the shared ones.  What a workgroup needs
// before it can ask for anything else comes first: it fetches that in one go.
struct PartsSide {
  DivU by_slots, by_groups;
  int n_slots, tiles_per_wg, row_groups, rows;  // rows: query rows of a sequence, or of the batch
  int slot0, shared;           // first record slot
  int res_cost;                // a residual head's time per token, a plain one's being 16; 0: every head takes n_slots
                               // workgroups (shared parts only)
  int by_cost;                 // the workgroups of a (sequence, chunk) go to the heads in the order of their cost
  int part_base[kMaxParts];    // first slot of each part, from 0; INT32_MAX past the last
  PartsPart part[kMaxParts];
};

// One launch: workgroups 0 .. shared_wgs - 1 take the shared parts, the others those of single sequences.
struct PartsParams {
  uint32_t shared_wgs;
  DivU by_hkv, by_topk;
  int hkv, hq, G, g_shift, n_blocks, block, pos, bsize, topk, tail_cap, n_slots_total;
  const void* q;               // [batch][hq][d]
  float* ws;                   // records [batch][hkv][n_slots_total][G][d + 4]
  const void* tail_k;          // [batch][hkv][tail_cap][d]
  const void* tail_v;
  int* shared_counts;          // [hkv] out: record slots that a head of the shared part fills (res_cost > 0)
  float wres[3], scale_log2;
  PartsSide side[2];           // single sequences, shared
  int batch, d;
  int res_ppm, n_rates;
  int rates_ppm[kMaxRates];
  bool tokres, bf16, coef8;
  int cols;                    // query rows of a workgroup of the shared parts: 16, 32, 64 or 128
};

struct PartsMergeParams {
  DivU by_hkv;
  const float* ws;             // records [batch][hkv][n_slots_total][G][d + 4]
  const int* shared_counts;    // [hkv] slots in use after the first own_slots, or null: all of n_slots_total
  int own_slots, n_slots_total, batch, hq, hkv, G, g_shift, d;
  bool bf16;
  void* out;                   // [batch][hq][d]
};

hipError_t launch_rope_append(const RopeParams& P, hipStream_t s);
hipError_t launch_key_bounds(const BoundsParams& P, hipStream_t s);
hipError_t launch_block_select(const SelectParams& P, hipStream_t s);
hipError_t launch_parts_f32_d64(const PartsParams& P, hipStream_t s);   // records of one launch's parts
hipError_t launch_parts_f32_d128(const PartsParams& P, hipStream_t s);
hipError_t launch_parts_bf16_d64(const PartsParams& P, hipStream_t s);
hipError_t launch_parts_bf16_d128(const PartsParams& P, hipStream_t s);
hipError_t launch_parts_c8_d64(const PartsParams& P, hipStream_t s);
hipError_t launch_parts_c8_d128(const PartsParams& P, hipStream_t s);
hipError_t launch_parts_merge(const PartsMergeParams& P, hipStream_t s);

}  // namespace fdkv
