// Attention over pages of 4 bits: what its kernels share (ptc_attn4_few.cu:
// requests of few query rows; ptc_attn4.cu: the others, and the C entry point).
#pragma once

#include "ptc_attn.cuh"
#include "ptc_kv4.cuh"

namespace ptc {

// Most query rows (new tokens times query heads of a key head) of a request that
// k_attn4_few takes: as many as its registers hold.  Up to there it is the faster, us
// by it and by the tile kernel:
//   rows a request                                            8        16        24        32
//   12 requests over 32K to 131K, heads of 128        113  289  151  295  212  297  215  303
//                                 heads of 64          75  239   95  234  127  235  131  227
//   rows a request                                            4        12        20        32
//   64 requests over 1.1K to 12K, heads of 128         81  206  115  220  169  225  175  231
//                                 heads of 64          55  141   70  145  105  148  108  150
//   one request over 1,012, heads of 128               10   18            16   22   19   25
//                           heads of 64                 9   16            14   19   16   21
// The tile kernel takes 308 and 310 us for 40 and 64 rows of the first, 222 and 224 for 36
// and 64 of the second.
constexpr uint32_t kFew4Rows = 32;
constexpr uint32_t kFew4MaxCtas = 512;
constexpr uint32_t kMost4 = 0x7FFFFF00u;  // tokens of a request: positions are signed 32-bit numbers

// Workspace of k_attn4_few for requests of up to `rows` rows, and its launch.
size_t few4_ws(uint32_t head_dim, uint32_t rows);
ptc_status launch_few4(const AttnArgs& a, uint32_t rows, char* ws, bool bf16, cudaStream_t s);

}  // namespace ptc
