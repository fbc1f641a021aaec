// Attention over pages of 4 bits: what its kernels share (ptc_attn4_few.cu:
// requests of few query rows; ptc_attn4.cu: the others, and the C entry point).
#pragma once

#include "ptc_attn.cuh"
#include "ptc_kv4.cuh"

namespace ptc {

// Most query rows (new tokens times query heads of a key head) of a request that
// k_attn4_few takes.
constexpr uint32_t kFew4Rows = 16;
constexpr uint32_t kFew4MaxCtas = 512;
constexpr uint32_t kMost4 = 0x7FFFFF00u;  // tokens of a request: positions are signed 32-bit numbers

struct Few4Args {
  KvView kv;
  const char* q;
  int64_t q_tok, q_head;
  const uint64_t* tok_off;
  uint64_t n_tok;
  uint32_t n_q_heads, G, max_q_len;
  float scale;
  char* out;
  float* lse;
  uint32_t* arrived;  // parts of the split tile that begins in CTA c
  float* part;        // unnormalised rows of split tiles: [2 * ctas][rows][64 or 128]
  float2* part_ml;    // their maxima (in powers of two) and sums
  uint32_t ctas;
  uint32_t div_mul, div_shift;  // key / B
  uint32_t* status;
};

// CTAs of a call, and its workspace behind the status word.
uint32_t few4_ctas(uint32_t head_dim, uint32_t rows);
size_t few4_ws(uint32_t head_dim, uint32_t rows);
void few4_place(Few4Args& a, uint32_t rows, char* ws);
ptc_status launch_few4(Few4Args& a, uint32_t rows, bool bf16, cudaStream_t s);

}  // namespace ptc
