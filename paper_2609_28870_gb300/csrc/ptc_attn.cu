// Attention of new tokens over paged keys and values (ptc_paged_attention).
#include <cmath>

#include "ptc_kv.cuh"

namespace ptc {
namespace {

struct AttnArgs {
  KvView kv;
  const char* q;
  int64_t q_tok, q_head;
  const uint64_t* tok_off;
  uint64_t n_tok;
  uint32_t n_q_heads, G, max_q_len;
  float scale;
  char* out;
  float* lse;
  const float* mass_in;
  float* mass_out;
  uint64_t mass_stride;
  uint32_t* ok;  // 1 if the call's lists are sound
  uint32_t* status;
};

// One CTA looks the lists over; the other kernels do nothing if they are not sound.
__global__ void __launch_bounds__(1024) k_attn_check(AttnArgs a) {
  grid_dep_sync();
  bool bad = threadIdx.x == 0 && (a.tok_off[0] != 0 || a.tok_off[a.kv.n_req] != a.n_tok);
  for (uint32_t r = threadIdx.x; r < a.kv.n_req; r += 1024) {
    const uint64_t lo = a.tok_off[r], hi = a.tok_off[r + 1];
    bad |= lo > hi || hi > a.n_tok || hi - lo > a.max_q_len || !pages_hold(a.kv, r, a.kv.kv_len[r]);
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) {
    *a.ok = !bad;
    if (bad) report(a.status, PTC_ERR_INVALID_ARG);
  }
}

template <typename T>
__device__ __forceinline__ float to_f(T x) { return static_cast<float>(x); }

template <typename T>
__device__ __forceinline__ float dot8(const uint4& a, const uint4& b, float acc) {
  const T* x = reinterpret_cast<const T*>(&a);
  const T* y = reinterpret_cast<const T*>(&b);
#pragma unroll
  for (int i = 0; i < 8; ++i) acc = fmaf(to_f(x[i]), to_f(y[i]), acc);
  return acc;
}

// One warp a query row: lanes over 32 keys for the scores, over head_dim for
// the values, running maximum and sum in 32 bits.
template <typename T>
__global__ void __launch_bounds__(256) k_attn_rows(AttnArgs a) {
  grid_dep_sync();
  if (!*a.ok) return;
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t row = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= a.n_tok * a.n_q_heads) return;
  const uint64_t t = row / a.n_q_heads;
  const uint32_t hq = (uint32_t)(row % a.n_q_heads), h = hq / a.G;
  const uint32_t r = req_search(a.tok_off, 0, a.kv.n_req - 1, t);
  const int64_t n = a.kv.kv_len[r];
  const int64_t sees = n - (int64_t)(a.tok_off[r + 1] - t) + 1;
  const uint64_t p0 = a.kv.page_off[r];
  const char* q = a.q + 2 * ((int64_t)t * a.q_tok + hq * a.q_head);
  float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t j0 = 0; j0 < sees; j0 += 32) {
    const int64_t j = j0 + lane;
    float s = -INFINITY;
    int64_t vrow = 0;
    if (j < sees) {
      const uint32_t page = a.kv.page_ids[p0 + j / a.kv.B];
      if (page < a.kv.n_pages) {
        const char* k = a.kv.k + 2 * (page * a.kv.ks_page + h * a.kv.ks_head + (j % a.kv.B) * a.kv.ks_slot);
        vrow = page * a.kv.vs_page + h * a.kv.vs_head + (j % a.kv.B) * a.kv.vs_slot;
        s = 0.f;
        for (uint32_t d = 0; d < a.kv.D; d += 8)
          s = dot8<T>(*reinterpret_cast<const uint4*>(q + 2 * d), *reinterpret_cast<const uint4*>(k + 2 * d), s);
        s *= a.scale;
      } else {
        report(a.status, PTC_ERR_INVALID_ARG);
      }
    }
    float top = s;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
    const float mn = fmaxf(m, top), base = mn == -INFINITY ? 0.f : mn;
    const float keep = expf(m - base), p = expf(s - base);
    float sum = p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
    l = l * keep + sum;
    m = mn;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] *= keep;
    const int cnt = sees - j0 < 32 ? (int)(sees - j0) : 32;
    for (int x = 0; x < cnt; ++x) {
      const float px = __shfl_sync(kFull, p, x);
      const int64_t vx = __shfl_sync(kFull, vrow, x);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t d = lane + 32 * i;
        if (d < a.kv.D) acc[i] = fmaf(px, to_f(*reinterpret_cast<const T*>(a.kv.v + 2 * (vx + d))), acc[i]);
      }
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t d = lane + 32 * i;
    if (d < a.kv.D) reinterpret_cast<T*>(a.out)[row * a.kv.D + d] = static_cast<T>(acc[i] * inv);
  }
  if (lane == 0) a.lse[row] = l > 0.f ? m + logf(l) : -INFINITY;
}

// One thread a slot and key head: its weights over every row that sees it.
template <typename T>
__global__ void __launch_bounds__(128) k_attn_mass(AttnArgs a) {
  grid_dep_sync();
  if (!*a.ok) return;
  const uint32_t h = blockIdx.y;
  const uint64_t total = a.kv.page_off[a.kv.n_req] - a.kv.page_off[0];
  const uint64_t slot = (uint64_t)blockIdx.x * 128 + threadIdx.x;
  if (slot >= total * a.kv.B) return;
  const uint64_t page_at = a.kv.page_off[0] + slot / a.kv.B;
  const uint32_t r = req_search(a.kv.page_off, 0, a.kv.n_req - 1, page_at);
  const int64_t j = (int64_t)((page_at - a.kv.page_off[r]) * a.kv.B + slot % a.kv.B);
  const uint64_t at = h * a.mass_stride + page_at * a.kv.B + slot % a.kv.B;
  const int64_t n = a.kv.kv_len[r], t0 = a.tok_off[r], m = (int64_t)a.tok_off[r + 1] - t0;
  float sum = 0.f;
  if (j < n) {
    const uint32_t page = a.kv.page_ids[page_at];
    if (page < a.kv.n_pages) {
      const char* k = a.kv.k + 2 * (page * a.kv.ks_page + h * a.kv.ks_head + (j % a.kv.B) * a.kv.ks_slot);
      for (int64_t i = j > n - m ? j - (n - m) : 0; i < m; ++i)
        for (uint32_t g = 0; g < a.G; ++g) {
          const char* q = a.q + 2 * ((t0 + i) * a.q_tok + (h * a.G + g) * a.q_head);
          float s = 0.f;
          for (uint32_t d = 0; d < a.kv.D; d += 8)
            s = dot8<T>(*reinterpret_cast<const uint4*>(q + 2 * d), *reinterpret_cast<const uint4*>(k + 2 * d), s);
          sum += expf(s * a.scale - a.lse[(t0 + i) * a.n_q_heads + h * a.G + g]);
        }
    }
    if (a.mass_in) sum += a.mass_in[at];
  }
  a.mass_out[at] = sum;
}

template <typename T>
void launch(const AttnArgs& a, cudaStream_t s) {
  PTC_KERNEL("k_attn_check", s, k_attn_check, 1, 1024, 0, a);
  if (a.n_tok)
    PTC_KERNEL("k_attn_rows", s, k_attn_rows<T>, (uint32_t)((a.n_tok * a.n_q_heads + 7) / 8), 256, 0, a);
  if (a.mass_out && a.kv.n_page_ids)
    PTC_KERNEL("k_attn_mass", s, k_attn_mass<T>, dim3((uint32_t)((a.kv.n_page_ids * a.kv.B + 127) / 128), a.kv.H), 128,
               0, a);
}

}  // namespace
}  // namespace ptc

using namespace ptc;

extern "C" size_t ptc_paged_attention_workspace_bytes(uint32_t, uint64_t, uint32_t, uint32_t, uint32_t) {
  return 2 * kKvStatusBytes;
}

extern "C" ptc_status ptc_paged_attention(const ptc_paged_kv* kv, const void* q, const int64_t q_stride[2],
                                          const uint64_t* tok_off, uint64_t n_tok, uint32_t n_q_heads,
                                          uint32_t max_q_len, float scale, void* out, float* lse,
                                          const float* mass_in, float* mass_out, uint64_t mass_stride, void* ws,
                                          size_t ws_bytes, uint32_t* status, void* stream) {
  AttnArgs a{};
  const ptc_status st = kv_view(kv, &a.kv);
  if (st != PTC_OK) return st;
  if (!tok_off || !q_stride || n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return PTC_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale) || (n_tok && !kv->n_req)) return PTC_ERR_INVALID_ARG;
  if (n_tok > (uint64_t(1) << 31) || n_tok * n_q_heads > (uint64_t(1) << 31) || kv->n_page_ids * kv->block_size > (uint64_t(1) << 38))
    return PTC_ERR_OVERFLOW;
  if (mass_out ? mass_stride / kv->block_size < kv->n_page_ids : mass_in != nullptr) return PTC_ERR_INVALID_ARG;
  if (!ws_ok(ws, ws_bytes, 2 * kKvStatusBytes)) return PTC_ERR_WORKSPACE;
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
  a.mass_in = mass_in;
  a.mass_out = mass_out;
  a.mass_stride = mass_stride;
  a.ok = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + kKvStatusBytes);
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  if (kv->dtype == PTC_DTYPE_BF16) launch<__nv_bfloat16>(a, s);
  else launch<__half>(a, s);
  return kv_end(status, a.status, s);
}
