// Attention of new tokens over pages of 4 bits (ptc_kv4_attention): requests of
// few rows by k_attn4_few, others by the tile kernel of the 16-bit pages, whose
// tiles four warps make of the codes.
#include "ptc_attn4.cuh"
#include "ptc_attn_tiles.cuh"

namespace ptc {
namespace {

template <typename T, int NSLAB>
ptc_status launch_tiles4(const AttnArgs& a, const CUtensorMap (&m)[4], cudaStream_t s) {
  using Sh = TileShape<NSLAB, kFour>;
  constexpr int smem = Sh::kSmem, threads = Sh::kThreads;
  static std::atomic<uint64_t> ready{0};
  const auto kernel = k_attn_tiles<T, NSLAB, false, kFour>;
  if (!large_smem(kernel, smem, ready)) return PTC_ERR_CUDA;
  PTC_KERNEL("k_attn4_tiles", s, kernel, a.ctas, threads, smem, m[0], m[1], m[2], m[3], a);
  return PTC_OK;
}

template <typename T>
ptc_status launch4(const AttnArgs& a, cudaStream_t s) {
  constexpr bool bf16 = Weights<T>::kBf16;
  launch_plan(a, false, s);
  if (!a.n_tok) return PTC_OK;
  CUtensorMap m[4] = {};
  if (!tokens_map(&m[2], a, bf16, a.tq) || (a.tq32 && !tokens_map(&m[3], a, bf16, a.tq32))) return PTC_ERR_CUDA;
  return a.kv.D > 64 ? launch_tiles4<T, 2>(a, m, s) : launch_tiles4<T, 1>(a, m, s);
}

// Query rows of a request, or none of k_attn4_few's where there may be more than it takes.
uint32_t few_rows(uint32_t n_q_heads, uint32_t n_kv_heads, uint32_t max_q_len) {
  const uint64_t rows = (uint64_t)max_q_len * (n_kv_heads ? n_q_heads / n_kv_heads : 0);
  return rows <= kFew4Rows ? (uint32_t)rows : 0;
}

}  // namespace
}  // namespace ptc

using namespace ptc;

extern "C" size_t ptc_kv4_attention_workspace_bytes(uint32_t n_req, uint32_t n_q_heads, uint32_t n_kv_heads,
                                                    uint32_t head_dim, uint32_t max_q_len) {
  const uint32_t rows = few_rows(n_q_heads, n_kv_heads, max_q_len);
  return rows ? kKvStatusBytes + few4_ws(head_dim, rows) : attn_ws(n_req, tile_ctas(), head_dim, 0).total;
}

extern "C" ptc_status ptc_kv4_attention(const ptc_paged_kv* kv, const void* q, const int64_t q_stride[2],
                                        const uint64_t* tok_off, uint64_t n_tok, uint32_t n_q_heads, uint32_t max_q_len,
                                        float scale, void* out, float* lse, void* ws, size_t ws_bytes, uint32_t* status,
                                        void* stream) {
  AttnArgs a{};
  const ptc_status st = kv4_view(kv, &a.kv);
  if (st != PTC_OK) return st;
  const ptc_status fits = attn_call(a, kv, tok_off, n_tok, q_stride, n_q_heads, scale);
  if (fits != PTC_OK) return fits;
  if (n_tok > 0x7FFFFFFFu || n_tok * n_q_heads > (uint64_t(1) << 31) ||
      kv->n_page_ids > (uint64_t(1) << 38) / kv->block_size || kv->n_pages > 0x7FFFFFFFu)
    return PTC_ERR_OVERFLOW;
  if (!ws_ok(ws, ws_bytes, ptc_kv4_attention_workspace_bytes(kv->n_req, n_q_heads, kv->n_kv_heads, kv->head_dim, max_q_len)))
    return PTC_ERR_WORKSPACE;
  if (kv->n_req == 0) return PTC_OK;
  const ptc_status rows = attn_rows(a, q, q_stride, max_q_len, out, lse);
  if (rows != PTC_OK) return rows;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  const bool bf16 = kv->dtype == PTC_DTYPE_BF16;
  ptc_status run;
  if (const uint32_t few = few_rows(n_q_heads, kv->n_kv_heads, max_q_len)) {
    run = launch_few4(a, few, static_cast<char*>(ws) + kKvStatusBytes, bf16, s);
  } else {
    page_division(a.kv.B, &a.div_mul, &a.div_shift);
    attn_place(a, attn_ws(kv->n_req, tile_ctas(), kv->head_dim, 0), static_cast<char*>(ws));
    run = bf16 ? launch4<__nv_bfloat16>(a, s) : launch4<__half>(a, s);
  }
  if (run != PTC_OK) return run;
  return kv_end(status, a.status, s);
}
