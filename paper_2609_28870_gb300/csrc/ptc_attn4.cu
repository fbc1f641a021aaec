// Attention of new tokens over pages of 4 bits (ptc_kv4_attention): requests of
// few rows by k_attn4_few, others by the tile kernel of the 16-bit pages, whose
// tiles four warps make of the codes, or, where many query tiles read the same
// keys, over a copy of the call's pages in 16 bits.
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

// ------------------------------------------------------------------ a copy in 16 bits
// Taking a key tile's codes to 16 bits costs the tile kernel a fifth of the time of
// every query tile that reads it (what goes through shared memory: the products, 192
// KB a pair of tiles, 64 in 16 bits and twice 20 of codes), a copy of the pages once
// 672 bytes of HBM a key and value of 128.  Without the copy and with it, us:
//   one request over 28,701, 4 heads of 128 a key head, 4,096 tokens     1,504  1,292
//                                                       1,024; 512; 256  396 370; 220 224; 144 162
//   24 requests over 3,000, the same heads, 384; 256; 64 tokens each     483 471; 331 347; 114 165
//   24 ragged ones over up to 12,000, 1 to 1,024; 512; 256 tokens        329 295; 199 198; 134 146
//   the same, 2 heads of 64 a key head, 1 to 2,048; 1,024; 512           272 251; 153 153; 101 107
// So the longest request decides, and a mean keeps one chunk among many single tokens
// from a copy of them all.
constexpr uint64_t kCopyRows = 2048, kCopyMean = 384;  // fewest query rows of the longest request, and on average
constexpr uint64_t kCopyBytes = uint64_t(1) << 30;     // the largest copy
constexpr int kCopyThreads = 256;

struct CopyArgs {
  KvView kv;
  const uint64_t* tok_off;
  uint32_t* ids;
  char* k;
  char* v;
};

// A CTA has an entry of the page lists.  One that a request with new tokens needs
// becomes page i of the copy (a page that the cache does not have: none); the others'
// pages stay as they are, and nothing reads them.
template <typename T, int LANES>
__global__ void __launch_bounds__(kCopyThreads) k_kv4_copy(const __grid_constant__ CopyArgs a) {
  grid_dep_sync();
  __shared__ uint32_t s_id;
  const uint64_t i = blockIdx.x;
  const uint32_t B = a.kv.B, H = a.kv.H, D = a.kv.D;
  if (threadIdx.x == 0) {
    const uint32_t r = req_search(a.kv.page_off, 0, a.kv.n_req - 1, i);
    const uint64_t first = a.kv.page_off[r];
    const bool needed = i >= first && i < a.kv.page_off[r + 1] && (i - first) * B < a.kv.kv_len[r] &&
                        a.tok_off[r] < a.tok_off[r + 1];
    const uint32_t id = needed ? a.kv.page_ids[i] : kNone;
    s_id = id < a.kv.n_pages ? id : kNone;
    a.ids[i] = id < a.kv.n_pages ? (uint32_t)i : kNone;
  }
  __syncthreads();
  const uint32_t id = s_id, c = threadIdx.x % LANES;
  if (id == kNone || 8 * c >= D) return;
  constexpr uint32_t kAtOnce = kCopyThreads / LANES;
  const uint32_t rows = H * B;
#pragma unroll 2
  for (uint32_t x = threadIdx.x / LANES; x < rows; x += kAtOnce) {
    const uint32_t h = x / B, slot = x % B;
    const uint32_t* k = reinterpret_cast<const uint32_t*>(a.kv.k + id * a.kv.ks_page + h * a.kv.ks_head + slot * a.kv.ks_slot);
    const uint32_t* v = reinterpret_cast<const uint32_t*>(a.kv.v + id * a.kv.vs_page + h * a.kv.vs_head + slot * a.kv.vs_slot);
    const uint32_t kw = k[c], kp = k[LANES + c / 4], vw = v[c], vp = v[LANES + c / 4];
    const uint32_t ks = both_low(kp), kb = both_high(kp), vs = both_low(vp), vb = both_high(vp);
    const uint64_t to = 2 * ((i * rows + x) * D + 8 * c);
    *reinterpret_cast<uint4*>(a.k + to) = make_uint4(fma16x2<T>(pair4<T>(kw, 0), ks, kb), fma16x2<T>(pair4<T>(kw, 1), ks, kb),
                                                     fma16x2<T>(pair4<T>(kw, 2), ks, kb), fma16x2<T>(pair4<T>(kw, 3), ks, kb));
    *reinterpret_cast<uint4*>(a.v + to) = make_uint4(fma16x2<T>(pair4<T>(vw, 0), vs, vb), fma16x2<T>(pair4<T>(vw, 1), vs, vb),
                                                     fma16x2<T>(pair4<T>(vw, 2), vs, vb), fma16x2<T>(pair4<T>(vw, 3), vs, vb));
  }
}

// Bytes of the copy's keys, and of its values; 0 where there is none.
size_t copy_bytes(uint32_t n_req, uint32_t G, uint32_t n_kv_heads, uint32_t head_dim, uint32_t max_q_len, uint64_t n_tok,
                  uint64_t n_page_ids, uint32_t block_size) {
  if (!n_req || !n_page_ids || block_size % 8) return 0;
  if ((uint64_t)max_q_len * G < kCopyRows || n_tok * G < kCopyMean * n_req) return 0;
  const uint64_t page = 2ull * block_size * n_kv_heads * head_dim;
  if (!page || n_page_ids > kCopyBytes / 2 / page) return 0;  // (sizes are asked for before the cache is checked)
  return (page * n_page_ids + 255) / 256 * 256;
}

template <typename T>
ptc_status launch_copied(AttnArgs& a, char* ws, size_t bytes, cudaStream_t s) {
  CopyArgs c{a.kv, a.tok_off, reinterpret_cast<uint32_t*>(ws)};
  c.k = ws + (4 * a.kv.n_page_ids + 255) / 256 * 256;
  c.v = c.k + bytes;
  const uint32_t ctas = (uint32_t)a.kv.n_page_ids;
  if (a.kv.D <= 64) PTC_KERNEL("k_kv4_copy", s, (k_kv4_copy<T, 8>), ctas, kCopyThreads, 0, c);
  else PTC_KERNEL("k_kv4_copy", s, (k_kv4_copy<T, 16>), ctas, kCopyThreads, 0, c);
  a.kv.k = c.k;
  a.kv.v = c.v;
  a.kv.ks_slot = a.kv.vs_slot = a.kv.D;
  a.kv.ks_head = a.kv.vs_head = (int64_t)a.kv.B * a.kv.D;
  a.kv.ks_page = a.kv.vs_page = a.kv.H * a.kv.ks_head;
  a.kv.page_ids = c.ids;
  a.kv.n_pages = ctas;
  return launch_attention(a, Weights<T>::kBf16, s);
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
                                                    uint32_t head_dim, uint32_t max_q_len, uint64_t n_tok,
                                                    uint64_t n_page_ids, uint32_t block_size) {
  const uint32_t rows = few_rows(n_q_heads, n_kv_heads, max_q_len);
  if (rows) return kKvStatusBytes + few4_ws(head_dim, rows);
  const size_t all = attn_ws(n_req, tile_ctas(), head_dim, 0).total;
  const size_t copy = copy_bytes(n_req, n_kv_heads ? n_q_heads / n_kv_heads : 0, n_kv_heads, head_dim, max_q_len, n_tok,
                                 n_page_ids, block_size);
  return copy ? all + (4 * n_page_ids + 255) / 256 * 256 + 2 * copy : all;
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
  a.most = kMost4;
  if (n_tok > 0x7FFFFFFFu || n_tok * n_q_heads > (uint64_t(1) << 31) ||
      kv->n_page_ids > (uint64_t(1) << 38) / kv->block_size || kv->n_pages > 0x7FFFFFFFu)
    return PTC_ERR_OVERFLOW;
  if (!ws_ok(ws, ws_bytes, ptc_kv4_attention_workspace_bytes(kv->n_req, n_q_heads, kv->n_kv_heads, kv->head_dim, max_q_len, n_tok,
                                                             kv->n_page_ids, kv->block_size)))
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
    const AttnWs at = attn_ws(kv->n_req, tile_ctas(), kv->head_dim, 0);
    const size_t copy = copy_bytes(kv->n_req, a.G, kv->n_kv_heads, kv->head_dim, max_q_len, n_tok, kv->n_page_ids, kv->block_size);
    char* w = static_cast<char*>(ws);
    attn_place(a, at, w);
    page_division(a.kv.B, &a.div_mul, &a.div_shift);
    if (copy) run = bf16 ? launch_copied<__nv_bfloat16>(a, w + at.total, copy, s) : launch_copied<__half>(a, w + at.total, copy, s);
    else run = bf16 ? launch4<__nv_bfloat16>(a, s) : launch4<__half>(a, s);
  }
  if (run != PTC_OK) return run;
  return kv_end(status, a.status, s);
}
