// Paged keys and values: the write of new tokens (ptc_kv_append) and the
// eviction by accumulated attention weight (ptc_kv_evict).
#include "ptc_kv.cuh"

namespace ptc {
namespace {

// ------------------------------------------------------------------ append
// A copy: T rows of H * D values for k and for v, read and written once, so
// HBM bounds it.  A CTA takes `per` consecutive tokens; one thread a token
// finds the token's request and slot, then all threads move 16 bytes each.
constexpr int kApThreads = 256;
constexpr uint32_t kApMaxTok = 16;

struct AppendArgs {
  KvView kv;
  const char* kn;
  const char* vn;
  int64_t kn_tok, kn_head, vn_tok, vn_head;
  const uint64_t* tok_off;
  uint64_t n_tok;
  uint32_t per;
  uint32_t* status;
};

__global__ void __launch_bounds__(kApThreads) k_kv_append(AppendArgs a) {
  grid_dep_sync();
  __shared__ int64_t s_k[kApMaxTok], s_v[kApMaxTok];  // element offset of head 0, or -1
  const uint64_t t0 = (uint64_t)blockIdx.x * a.per;
  const uint32_t nt = (uint32_t)(a.n_tok - t0 < a.per ? a.n_tok - t0 : a.per);
  if (blockIdx.x == 0) {
    bool bad = threadIdx.x == 0 && (a.tok_off[0] != 0 || a.tok_off[a.kv.n_req] != a.n_tok);
    for (uint32_t r = threadIdx.x; r < a.kv.n_req; r += kApThreads) bad |= a.tok_off[r] > a.tok_off[r + 1];
    if (bad) report(a.status, PTC_ERR_INVALID_ARG);
  }
  if (threadIdx.x < nt) {
    const uint64_t t = t0 + threadIdx.x;
    const uint32_t r = req_search(a.tok_off, 0, a.kv.n_req - 1, t);
    const uint64_t lo = a.tok_off[r], hi = a.tok_off[r + 1];
    const uint64_t n = a.kv.kv_len[r];
    int64_t k = -1, v = -1;
    if (lo <= t && t < hi && hi <= a.n_tok && hi - lo <= n && pages_hold(a.kv, r, n)) {
      const uint64_t j = n - (hi - t);
      const uint32_t page = a.kv.page_ids[a.kv.page_off[r] + j / a.kv.B];
      const int64_t slot = (int64_t)(j % a.kv.B);
      if (page < a.kv.n_pages) {
        k = (int64_t)page * a.kv.ks_page + slot * a.kv.ks_slot;
        v = (int64_t)page * a.kv.vs_page + slot * a.kv.vs_slot;
      }
    }
    if (k < 0) report(a.status, PTC_ERR_INVALID_ARG);
    s_k[threadIdx.x] = k;
    s_v[threadIdx.x] = v;
  }
  __syncthreads();
  const uint32_t chunks = a.kv.D / 8, row = a.kv.H * chunks;  // 16-byte pieces of a head, of a token
  for (uint32_t i = threadIdx.x; i < nt * row; i += kApThreads) {
    const uint32_t tok = i / row, c = i % row;
    const int64_t h = c / chunks, d = (c % chunks) * 8;
    if (s_k[tok] < 0) continue;
    const int64_t t = (int64_t)(t0 + tok);
    const uint4 kx = *reinterpret_cast<const uint4*>(a.kn + 2 * (t * a.kn_tok + h * a.kn_head + d));
    const uint4 vx = *reinterpret_cast<const uint4*>(a.vn + 2 * (t * a.vn_tok + h * a.vn_head + d));
    *reinterpret_cast<uint4*>(a.kv.k + 2 * (s_k[tok] + h * a.kv.ks_head + d)) = kx;
    *reinterpret_cast<uint4*>(a.kv.v + 2 * (s_v[tok] + h * a.kv.vs_head + d)) = vx;
  }
}

// ------------------------------------------------------------------ evict
struct EvictArgs {
  KvView kv;
  const float* mass;
  uint64_t mass_stride;
  uint32_t n_keep, n_sink, n_recent, max_kv_len;
  const uint32_t* dst_ids;
  const uint64_t* dst_off;
  uint64_t n_dst_ids;
  uint32_t* keep;
  uint32_t* new_len;
  float* new_mass;
  uint64_t new_mass_stride;
  uint32_t* ok;  // per request: 1 if its lists are sound
  uint32_t* status;
};

// Weights as integers in the same order: NaN lowest, -0 equal to 0.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelThreads = 1024;
constexpr int kSelBins = 2048;

// One CTA a request and key head: the threshold weight by a radix search
// (11, 11 and 10 bits, histograms in shared memory), then the kept positions
// in order by a scan.
__global__ void __launch_bounds__(kSelThreads) k_evict_select(EvictArgs a) {
  grid_dep_sync();
  __shared__ uint32_t s_hist[kSelBins];
  __shared__ uint32_t s_warp[32], s_warp2[32];
  __shared__ uint32_t s_bin, s_above;
  const uint32_t h = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t n = a.kv.kv_len[r], b = n < a.n_keep ? n : a.n_keep;
  const uint64_t d0 = a.dst_off[r], d1 = a.dst_off[r + 1];
  const bool ok = n <= a.max_kv_len && pages_hold(a.kv, r, n) && d0 <= d1 && d1 <= a.n_dst_ids &&
                  b <= (d1 - d0) * a.kv.B;
  if (h == 0 && tid == 0) {
    a.ok[r] = ok;
    a.new_len[r] = b;
    if (!ok) report(a.status, PTC_ERR_INVALID_ARG);
  }
  if (!ok) return;
  uint32_t* keep = a.keep + ((uint64_t)r * a.kv.H + h) * a.n_keep;
  for (uint32_t i = b + tid; i < a.n_keep; i += kSelThreads) keep[i] = kNone;
  if (b == n) {
    for (uint32_t i = tid; i < n; i += kSelThreads) keep[i] = i;
    return;
  }
  const float* w = a.mass + h * a.mass_stride + a.kv.page_off[r] * a.kv.B;
  const uint32_t lo = a.n_sink, hi = n - a.n_recent;
  uint32_t need = b - a.n_sink - a.n_recent;
  // the need-th largest of [lo, hi): prefix holds the bits settled so far
  uint32_t prefix = 0, mask = 0;
  if (need) {
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
      for (uint32_t i = tid; i < kSelBins; i += kSelThreads) s_hist[i] = 0;
      __syncthreads();
      for (uint32_t j = lo + tid; j < hi; j += kSelThreads) {
        const uint32_t o = order_of(w[j]);
        if ((o & mask) == prefix) atomicAdd(&s_hist[(o >> shift) & ((1u << bits) - 1)], 1u);
      }
      __syncthreads();
      // bins from the top: thread t has bins 2047 - 2t and 2046 - 2t
      const uint32_t c0 = s_hist[kSelBins - 1 - 2 * tid], c1 = s_hist[kSelBins - 2 - 2 * tid];
      uint32_t x = c0 + c1;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(kFull, x, o);
        if (lane >= (uint32_t)o) x += y;
      }
      if (lane == 31) s_warp[warp] = x;
      __syncthreads();
      uint32_t before = x - c0 - c1;
      for (uint32_t i = 0; i < warp; ++i) before += s_warp[i];
      if (before < need && need <= before + c0) {
        s_bin = kSelBins - 1 - 2 * tid;
        s_above = before;
      } else if (before + c0 < need && need <= before + c0 + c1) {
        s_bin = kSelBins - 2 - 2 * tid;
        s_above = before + c0;
      }
      __syncthreads();
      prefix |= s_bin << shift;
      mask |= ((1u << bits) - 1) << shift;
      need -= s_above;
      __syncthreads();
    }
  } else {
    prefix = 0xFFFFFFFFu;  // above every weight
  }
  // kept: sinks, recent tokens, weights above the threshold, and the first `need` equal to it
  uint32_t kept = 0, ties = 0;
  for (uint32_t base = 0; base < n; base += kSelThreads) {
    const uint32_t j = base + tid;
    bool more = false, tie = false;
    if (j < n) {
      if (j < lo || j >= hi) {
        more = true;
      } else {
        const uint32_t o = order_of(w[j]);
        more = o > prefix;
        tie = o == prefix;
      }
    }
    const uint32_t bt = __ballot_sync(kFull, tie);
    if (lane == 0) s_warp2[warp] = __popc(bt);
    __syncthreads();
    uint32_t t_before = ties, t_all = ties;
    for (uint32_t i = 0; i < 32; ++i) {
      if (i < warp) t_before += s_warp2[i];
      t_all += s_warp2[i];
    }
    if (tie && t_before + __popc(bt & ((1u << lane) - 1)) < need) more = true;
    const uint32_t bk = __ballot_sync(kFull, more);
    if (lane == 0) s_warp[warp] = __popc(bk);
    __syncthreads();
    uint32_t k_before = kept, k_all = kept;
    for (uint32_t i = 0; i < 32; ++i) {
      if (i < warp) k_before += s_warp[i];
      k_all += s_warp[i];
    }
    if (more) keep[k_before + __popc(bk & ((1u << lane) - 1))] = j;
    kept = k_all;
    ties = t_all;
    __syncthreads();
  }
}

constexpr int kMvThreads = 256;
constexpr uint32_t kMvRows = 32;

// The move: kMvRows kept rows of one request and head a CTA.
__global__ void __launch_bounds__(kMvThreads) k_evict_move(EvictArgs a) {
  grid_dep_sync();
  const uint32_t h = blockIdx.y, r = blockIdx.z, i0 = blockIdx.x * kMvRows;
  if (!a.ok[r]) return;
  const uint32_t b = a.new_len[r], n = a.kv.kv_len[r];
  const uint64_t p0 = a.kv.page_off[r], d0 = a.dst_off[r], room = (a.dst_off[r + 1] - d0) * a.kv.B;
  const uint32_t* keep = a.keep + ((uint64_t)r * a.kv.H + h) * a.n_keep;
  if (blockIdx.x == 0)
    for (uint64_t i = b + threadIdx.x; i < room; i += kMvThreads) a.new_mass[h * a.new_mass_stride + d0 * a.kv.B + i] = 0.f;
  const uint32_t rows = i0 >= b ? 0 : (b - i0 < kMvRows ? b - i0 : kMvRows), chunks = a.kv.D / 8;
  for (uint32_t x = threadIdx.x; x < rows * chunks; x += kMvThreads) {
    const uint32_t i = i0 + x / chunks, d = (x % chunks) * 8;
    const uint32_t j = keep[i];
    if (j >= n) continue;
    const uint32_t ps = a.kv.page_ids[p0 + j / a.kv.B], pd = a.dst_ids[d0 + i / a.kv.B];
    if (ps >= a.kv.n_pages || pd >= a.kv.n_pages) {
      report(a.status, PTC_ERR_INVALID_ARG);
      continue;
    }
    const int64_t ss = j % a.kv.B, sd = i % a.kv.B;
    const int64_t kh = h * a.kv.ks_head + d, vh = h * a.kv.vs_head + d;
    const uint4 kx = *reinterpret_cast<const uint4*>(a.kv.k + 2 * (ps * a.kv.ks_page + ss * a.kv.ks_slot + kh));
    const uint4 vx = *reinterpret_cast<const uint4*>(a.kv.v + 2 * (ps * a.kv.vs_page + ss * a.kv.vs_slot + vh));
    *reinterpret_cast<uint4*>(a.kv.k + 2 * (pd * a.kv.ks_page + sd * a.kv.ks_slot + kh)) = kx;
    *reinterpret_cast<uint4*>(a.kv.v + 2 * (pd * a.kv.vs_page + sd * a.kv.vs_slot + vh)) = vx;
    if (d == 0)
      a.new_mass[h * a.new_mass_stride + d0 * a.kv.B + i] = a.mass[h * a.mass_stride + p0 * a.kv.B + j];
  }
}

size_t evict_bytes(uint32_t n_req) { return kKvStatusBytes + ((size_t)n_req * 4 + 255) / 256 * 256; }

}  // namespace
}  // namespace ptc

using namespace ptc;

extern "C" size_t ptc_kv_append_workspace_bytes(uint32_t) { return kKvStatusBytes; }

extern "C" ptc_status ptc_kv_append(const ptc_paged_kv* kv, const void* k_new, const void* v_new,
                                    const int64_t k_new_stride[2], const int64_t v_new_stride[2],
                                    const uint64_t* tok_off, uint64_t n_tok, void* ws, size_t ws_bytes,
                                    uint32_t* status, void* stream) {
  AppendArgs a{};
  const ptc_status st = kv_view(kv, &a.kv);
  if (st != PTC_OK) return st;
  if (!tok_off || !k_new_stride || !v_new_stride || (n_tok && !kv->n_req)) return PTC_ERR_INVALID_ARG;
  if (n_tok > (uint64_t(1) << 31)) return PTC_ERR_OVERFLOW;
  if (!ws_ok(ws, ws_bytes, kKvStatusBytes)) return PTC_ERR_WORKSPACE;
  if (n_tok == 0) return PTC_OK;
  if (!aligned16(k_new) || !aligned16(v_new)) return PTC_ERR_INVALID_ARG;
  const uint32_t ext[2] = {(uint32_t)n_tok, kv->n_kv_heads};
  for (int i = 0; i < 2; ++i)
    if (!stride_ok(k_new_stride[i], ext[i]) || !stride_ok(v_new_stride[i], ext[i])) return PTC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  a.kn = static_cast<const char*>(k_new);
  a.vn = static_cast<const char*>(v_new);
  a.kn_tok = stride_of(k_new_stride[0], ext[0]);
  a.kn_head = stride_of(k_new_stride[1], ext[1]);
  a.vn_tok = stride_of(v_new_stride[0], ext[0]);
  a.vn_head = stride_of(v_new_stride[1], ext[1]);
  a.tok_off = tok_off;
  a.n_tok = n_tok;
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  const uint64_t per = (n_tok + 4 * num_sms() - 1) / (4 * num_sms());
  a.per = (uint32_t)(per < kApMaxTok ? per : kApMaxTok);
  PTC_KERNEL("k_kv_append", s, k_kv_append, (uint32_t)((n_tok + a.per - 1) / a.per), kApThreads, 0, a);
  return kv_end(status, a.status, s);
}

extern "C" size_t ptc_kv_evict_workspace_bytes(uint32_t n_req, uint32_t, uint32_t) { return evict_bytes(n_req); }

extern "C" ptc_status ptc_kv_evict(const ptc_paged_kv* kv, const float* mass, uint64_t mass_stride, uint32_t n_keep,
                                   uint32_t n_sink, uint32_t n_recent, uint32_t max_kv_len,
                                   const uint32_t* dst_page_ids, const uint64_t* dst_page_off,
                                   uint64_t n_dst_page_ids, uint32_t* keep_out, uint32_t* new_len_out,
                                   float* new_mass_out, uint64_t new_mass_stride, void* ws, size_t ws_bytes,
                                   uint32_t* status, void* stream) {
  EvictArgs a{};
  const ptc_status st = kv_view(kv, &a.kv);
  if (st != PTC_OK) return st;
  if (n_keep < 1 || (uint64_t)n_sink + n_recent > n_keep) return PTC_ERR_INVALID_ARG;
  if (!dst_page_off || (n_dst_page_ids && !dst_page_ids)) return PTC_ERR_INVALID_ARG;
  if (n_keep > (1u << 30) || max_kv_len > (1u << 31)) return PTC_ERR_OVERFLOW;
  if (!ws_ok(ws, ws_bytes, evict_bytes(kv->n_req))) return PTC_ERR_WORKSPACE;
  if (kv->n_req == 0) return PTC_OK;
  if ((kv->n_page_ids && !mass) || (n_dst_page_ids && (!new_mass_out || new_mass_out == mass))) return PTC_ERR_INVALID_ARG;
  if (!keep_out || !new_len_out) return PTC_ERR_INVALID_ARG;
  if (mass_stride / kv->block_size < kv->n_page_ids || new_mass_stride / kv->block_size < n_dst_page_ids)
    return PTC_ERR_INVALID_ARG;
  if (kv->n_req > 65535) return PTC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  a.mass = mass;
  a.mass_stride = mass_stride;
  a.n_keep = n_keep;
  a.n_sink = n_sink;
  a.n_recent = n_recent;
  a.max_kv_len = max_kv_len;
  a.dst_ids = dst_page_ids;
  a.dst_off = dst_page_off;
  a.n_dst_ids = n_dst_page_ids;
  a.keep = keep_out;
  a.new_len = new_len_out;
  a.new_mass = new_mass_out;
  a.new_mass_stride = new_mass_stride;
  a.ok = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + kKvStatusBytes);
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  PTC_KERNEL("k_evict_select", s, k_evict_select, dim3(kv->n_kv_heads, kv->n_req), kSelThreads, 0, a);
  const uint32_t most = n_keep < max_kv_len ? n_keep : max_kv_len;
  const uint32_t gx = most ? (most + kMvRows - 1) / kMvRows : 1;
  PTC_KERNEL("k_evict_move", s, k_evict_move, dim3(gx, kv->n_kv_heads, kv->n_req), kMvThreads, 0, a);
  return kv_end(status, a.status, s);
}
