// Attention over pages of 4 bits: what its kernels share (ptc_attn4_few.cu:
// requests of few query rows; ptc_attn4.cu: the others, and the C entry point).
#pragma once

#include "ptc_attn.cuh"
#include "ptc_kv4.cuh"

namespace ptc {

// Most query rows (new tokens times query heads of a key head) of a request that
// k_attn4_few takes.
constexpr uint32_t kFew4Rows = 32;
constexpr uint32_t kFew4MaxCtas = 512;
constexpr uint32_t kMost4 = 0x7FFFFF00u;  // tokens of a request: positions are signed 32-bit numbers

// Workspace of k_attn4_few for requests of up to `rows` rows, and its launch.
size_t few4_ws(uint32_t head_dim, uint32_t rows);
ptc_status launch_few4(const AttnArgs& a, uint32_t rows, char* ws, bool bf16, cudaStream_t s);

}  // namespace ptc
