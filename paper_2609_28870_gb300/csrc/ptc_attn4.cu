// Attention of new tokens over pages of 4 bits (ptc_kv4_attention).
#include <cmath>

#include "ptc_attn4.cuh"

namespace ptc {
namespace {

struct Attn4Args {
  KvView kv;
  const char* q;
  int64_t q_tok, q_head;
  const uint64_t* tok_off;
  uint64_t n_tok;
  uint32_t n_q_heads, G, max_q_len;
  float scale;
  char* out;
  float* lse;
  uint32_t* status;
};

constexpr int kOneWarps = 4;

// A warp has one query head of one token.  For 32 keys at a time a lane takes a
// key's product, then each lane adds up four channels of the 32 values.
template <typename T>
__global__ void __launch_bounds__(32 * kOneWarps) k_attn4_rows(const Attn4Args a) {
  grid_dep_sync();
  using H = Half16<T>;
  __shared__ float s_q[kOneWarps][128];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, D = a.kv.D, Dp = padded4(D);
  if (blockIdx.x == 0) {
    bool bad = threadIdx.x == 0 && (a.tok_off[0] != 0 || a.tok_off[a.kv.n_req] != a.n_tok);
    for (uint32_t r = threadIdx.x; r < a.kv.n_req; r += 32 * kOneWarps)
      bad |= a.tok_off[r] > a.tok_off[r + 1] || a.tok_off[r + 1] - a.tok_off[r] > a.max_q_len || !pages_hold(a.kv, r, a.kv.kv_len[r]);
    if (bad) report(a.status, PTC_ERR_INVALID_ARG);
  }
  const uint64_t row = (uint64_t)blockIdx.x * kOneWarps + warp;
  if (row >= a.n_tok * a.n_q_heads) return;
  const uint64_t t = row / a.n_q_heads;
  const uint32_t g = (uint32_t)(row % a.n_q_heads), h = g / a.G;
  const uint32_t r = req_search(a.tok_off, 0, a.kv.n_req - 1, t);
  const uint64_t lo = a.tok_off[r], hi = a.tok_off[r + 1], n = a.kv.kv_len[r];
  if (!(lo <= t && t < hi && hi <= a.n_tok && pages_hold(a.kv, r, n))) return;
  const T* q = reinterpret_cast<const T*>(a.q) + t * a.q_tok + g * a.q_head;
  for (uint32_t d = lane; d < Dp; d += 32) s_q[warp][d] = d < D ? H::get(q[d]) * a.scale : 0.f;
  __syncwarp();
  const int64_t sees = (int64_t)n - (int64_t)(hi - t) + 1;
  float top = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t j0 = 0; j0 < sees; j0 += 32) {
    const int64_t j = j0 + lane;
    const char* v = nullptr;
    float s = -INFINITY;
    if (j < sees) {
      const uint32_t id = a.kv.page_ids[a.kv.page_off[r] + j / a.kv.B];
      const int64_t slot = j % a.kv.B;
      if (id < a.kv.n_pages) {
        const uint32_t* k = reinterpret_cast<const uint32_t*>(a.kv.k + id * a.kv.ks_page + h * a.kv.ks_head + slot * a.kv.ks_slot);
        v = a.kv.v + id * a.kv.vs_page + h * a.kv.vs_head + slot * a.kv.vs_slot;
        s = 0.f;
        for (uint32_t i = 0; 8 * i < D; ++i) {
          const uint32_t w = k[i], p = k[Dp / 8 + i / 4], sc = both_low(p), b = both_high(p);
          for (int x = 0; x < 4; ++x) {
            const float2 y = H::get2(fma16x2<T>(pair4<T>(w, x), sc, b));
            s = fmaf(y.x, s_q[warp][8 * i + 2 * x], s);
            s = fmaf(y.y, s_q[warp][8 * i + 2 * x + 1], s);
          }
        }
      } else {
        report(a.status, PTC_ERR_INVALID_ARG);
      }
    }
    float mx = s;
    for (int x = 16; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, x));
    mx = fmaxf(mx, top);
    const float f = top == -INFINITY ? 0.f : exp2f((top - mx) * kLog2e), p = s == -INFINITY ? 0.f : exp2f((s - mx) * kLog2e);
    top = mx;
    l = l * f + p;
    for (int x = 0; x < 4; ++x) o[x] *= f;
    for (int y = 0; y < 32; ++y) {
      const float w = __shfl_sync(kFull, p, y);
      const char* at = reinterpret_cast<const char*>(__shfl_sync(kFull, reinterpret_cast<uint64_t>(v), y));
      if (!at || 4 * lane >= D) continue;
      const uint32_t* words = reinterpret_cast<const uint32_t*>(at);
      const uint32_t c = words[lane / 2], par = words[Dp / 8 + lane / 8], sc = both_low(par), b = both_high(par);
      const float2 a0 = H::get2(fma16x2<T>(pair4<T>(c >> (lane & 1 ? 8 : 0), 0), sc, b));
      const float2 a1 = H::get2(fma16x2<T>(pair4<T>(c >> (lane & 1 ? 8 : 0), 1), sc, b));
      o[0] = fmaf(w, a0.x, o[0]);
      o[1] = fmaf(w, a0.y, o[1]);
      o[2] = fmaf(w, a1.x, o[2]);
      o[3] = fmaf(w, a1.y, o[3]);
    }
  }
  for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(kFull, l, x);
  const uint64_t at = t * a.n_q_heads + g;
  if (lane == 0) a.lse[at] = sees > 0 ? top + logf(l) : -INFINITY;
  T* out = reinterpret_cast<T*>(a.out) + at * D;
  for (int x = 0; x < 4; ++x)
    if (4 * lane + x < D) out[4 * lane + x] = H::put(sees > 0 ? o[x] / l : 0.f);
}

}  // namespace
}  // namespace ptc

using namespace ptc;

namespace {
// Query rows of a request, or none of k_attn4_few's where there may be more than it takes.
uint32_t few_rows(uint32_t n_q_heads, uint32_t n_kv_heads, uint32_t max_q_len) {
  const uint64_t rows = (uint64_t)max_q_len * (n_kv_heads ? n_q_heads / n_kv_heads : 0);
  return rows <= kFew4Rows ? (uint32_t)rows : 0;
}
}  // namespace

extern "C" size_t ptc_kv4_attention_workspace_bytes(uint32_t, uint32_t n_q_heads, uint32_t n_kv_heads, uint32_t head_dim,
                                                    uint32_t max_q_len) {
  const uint32_t rows = few_rows(n_q_heads, n_kv_heads, max_q_len);
  return kKvStatusBytes + (rows ? few4_ws(head_dim, rows) : 0);
}

extern "C" ptc_status ptc_kv4_attention(const ptc_paged_kv* kv, const void* q, const int64_t q_stride[2],
                                        const uint64_t* tok_off, uint64_t n_tok, uint32_t n_q_heads, uint32_t max_q_len,
                                        float scale, void* out, float* lse, void* ws, size_t ws_bytes, uint32_t* status,
                                        void* stream) {
  Attn4Args a{};
  const ptc_status st = kv4_view(kv, &a.kv);
  if (st != PTC_OK) return st;
  if (!tok_off || !q_stride || n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return PTC_ERR_INVALID_ARG;
  if (n_q_heads / kv->n_kv_heads > PTC_MAX_GROUP) return PTC_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale) || (n_tok && !kv->n_req)) return PTC_ERR_INVALID_ARG;
  if (!std::isfinite(scale * kLog2e)) return PTC_ERR_INVALID_ARG;
  if (n_tok > 0x7FFFFFFFu || n_tok * n_q_heads > (uint64_t(1) << 31) ||
      kv->n_page_ids > (uint64_t(1) << 38) / kv->block_size)
    return PTC_ERR_OVERFLOW;
  if (kv->n_pages > 0x7FFFFFFFu) return PTC_ERR_OVERFLOW;
  if (!ws_ok(ws, ws_bytes, ptc_kv4_attention_workspace_bytes(kv->n_req, n_q_heads, kv->n_kv_heads, kv->head_dim, max_q_len)))
    return PTC_ERR_WORKSPACE;
  if (kv->n_req == 0) return PTC_OK;
  if (n_tok && (!aligned16(q) || !aligned16(out) || !lse)) return PTC_ERR_INVALID_ARG;
  const uint32_t ext[2] = {(uint32_t)n_tok, n_q_heads};
  for (int i = 0; i < 2; ++i)
    if (!stride_ok(q_stride[i], ext[i])) return PTC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  a.q = static_cast<const char*>(q);
  a.q_tok = stride_of(q_stride[0], ext[0]);
  a.q_head = stride_of(q_stride[1], ext[1]);
  a.tok_off = tok_off;
  a.n_tok = n_tok;
  a.n_q_heads = n_q_heads;
  a.G = n_q_heads / kv->n_kv_heads;
  a.max_q_len = max_q_len;
  a.scale = scale;
  a.out = static_cast<char*>(out);
  a.lse = lse;
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  if (const uint32_t few = few_rows(n_q_heads, kv->n_kv_heads, max_q_len)) {
    Few4Args f{};
    f.kv = a.kv;
    f.q = a.q;
    f.q_tok = a.q_tok;
    f.q_head = a.q_head;
    f.tok_off = a.tok_off;
    f.n_tok = a.n_tok;
    f.n_q_heads = a.n_q_heads;
    f.G = a.G;
    f.max_q_len = max_q_len;
    f.scale = scale;
    f.out = a.out;
    f.lse = a.lse;
    f.status = a.status;
    few4_place(f, few, static_cast<char*>(ws) + kKvStatusBytes);
    const ptc_status run = launch_few4(f, few, kv->dtype == PTC_DTYPE_BF16, s);
    return run != PTC_OK ? run : kv_end(status, a.status, s);
  }
  const uint64_t rows = n_tok * n_q_heads;
  const uint32_t ctas = rows ? (uint32_t)((rows + kOneWarps - 1) / kOneWarps) : 1;
  if (kv->dtype == PTC_DTYPE_BF16) PTC_KERNEL("k_attn4_rows", s, k_attn4_rows<__nv_bfloat16>, ctas, 32 * kOneWarps, 0, a);
  else PTC_KERNEL("k_attn4_rows", s, k_attn4_rows<__half>, ctas, 32 * kOneWarps, 0, a);
  return kv_end(status, a.status, s);
}
