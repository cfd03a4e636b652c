// Parameter blocks and launchers of exact rows before their compression: the
// attention of a prompt, pages of rows, decode over pages (internal to libfdkv).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "divu.h"

namespace fdkv {

// causal attention of packed prompts (prompt.hip)
constexpr int kPromptRows = 128;    // query rows (token, head of the group) of a workgroup
struct PromptParams {
  DivU by_hkv;
  const void* q;               // [n_tokens][hq][d], q_stride bytes a token
  const void* k;               // [..][hkv][..][d]: bytes from sequence to sequence, head to head, row to row
  const void* v;
  int64_t q_stride, k_seq, k_head, k_row, v_seq, v_head, v_row;
  const int32_t* q_starts;     // [batch + 1]
  const int32_t* k_starts;     // [batch] or null
  const int32_t* k_lens;       // [batch]
  void* out;                   // [n_tokens][hq][d]
  float* ws;                   // records [splits][n_tokens][hq][d + 4]
  float scale_log2;
  int n_tokens, batch, hq, hkv, g_shift, rows, d, splits, tiles;
  int cut;                     // tiles of query rows that are taken from the last on, the others from the first on
  bool bf16;
};

// pages of rows (pages.hip)
struct PageParams {
  void* k;                     // [n_pages][hkv][page][d]
  void* v;
  uint8_t* k_exp;              // [n_pages][hkv][page], rows in E4M3
  uint8_t* v_exp;
  const int32_t* table;        // [batch][max_pages]
  int n_pages, log_page, batch, max_pages, hkv, d;
  bool bf16, coef8;
};
struct PageRowsParams {
  DivU by_heads;               // by 2 hkv
  PageParams pg;
  void* rows_k;                // [n_tokens][hkv][d]: read by a write, written by a read
  void* rows_v;
  int64_t k_tok, k_head, v_tok, v_head;  // bytes from token to token, head to head
  const int32_t* seqs;         // [n_tokens] or null (token i is of sequence i)
  const int32_t* rows;         // [n_tokens]
  int n_tokens;
};

// decode over pages (paged.hip)
constexpr int kPagedChunkMost = 2048;  // tokens of a workgroup, at most (128 pages of 16)
struct PagedParams {
  DivU by_hkv, by_chunks, by_chunk;  // by hkv, n_chunks, chunk
  PageParams pg;
  const int32_t* lens;         // [batch]
  const void* q;               // [batch][hq][d]
  void* out;                   // [batch][hq][d]
  float* ws;                   // records [batch][hkv][n_chunks][G][d + 4]
  const float* more;           // records of other tokens, [batch][hkv][n_more][G][d + 4]
  float scale_log2;
  int max_len, chunk, n_chunks, n_more, hq, g_shift;
};

hipError_t launch_prompt_attn(const PromptParams& P, hipStream_t s);
hipError_t launch_page_write(const PageRowsParams& P, hipStream_t s);
hipError_t launch_page_read(const PageRowsParams& P, hipStream_t s);
hipError_t launch_paged_attn(const PagedParams& P, hipStream_t s);

}  // namespace fdkv
