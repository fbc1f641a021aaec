// What the calls on paged keys and values share: the device view of the
// cache, the stream-ordered status word and the host-side argument checks.
#pragma once

#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ptc_internal.h"

namespace ptc {

// The cache as kernels see it; strides in elements.
struct KvView {
  char* k;
  char* v;
  int64_t ks_page, ks_head, ks_slot;
  int64_t vs_page, vs_head, vs_slot;
  const uint32_t* page_ids;
  const uint64_t* page_off;
  const uint32_t* kv_len;
  uint64_t n_page_ids;
  uint32_t n_pages, n_req, B, H, D;
};

// A kernel's report: the larger of the codes that its threads meet stays.
__device__ __forceinline__ void report(uint32_t* status, uint32_t code) { atomicMax(status, code); }

// Whether request r's page list is sound and holds n tokens.
__device__ __forceinline__ bool pages_hold(const KvView& kv, uint32_t r, uint64_t n) {
  const uint64_t a = kv.page_off[r], b = kv.page_off[r + 1];
  return a <= b && b <= kv.n_page_ids && n <= (b - a) * kv.B;
}

inline bool stride_ok(int64_t stride, uint32_t extent) {
  // tensor maps hold strides below 2^40 bytes
  return extent <= 1 || (stride > 0 && stride % 8 == 0 && stride < (int64_t(1) << 39));
}
inline int64_t stride_of(int64_t stride, uint32_t extent) { return extent <= 1 ? 8 : stride; }
inline bool aligned16(const void* p) { return p != nullptr && ((uintptr_t)p & 15) == 0; }

// The host-side checks of a ptc_paged_kv, and its device view.
inline ptc_status kv_view(const ptc_paged_kv* kv, KvView* o) {
  if (!kv) return PTC_ERR_INVALID_ARG;
  if (kv->dtype != PTC_DTYPE_BF16 && kv->dtype != PTC_DTYPE_FP16) return PTC_ERR_INVALID_ARG;
  if (kv->block_size < 1 || kv->block_size > PTC_MAX_BLOCK_SIZE || kv->n_kv_heads < 1 || kv->n_kv_heads > 65535)
    return PTC_ERR_INVALID_ARG;
  if (kv->head_dim < 16 || kv->head_dim > PTC_MAX_HEAD_DIM || kv->head_dim % 8) return PTC_ERR_INVALID_ARG;
  if (!kv->page_off || (kv->n_req && !kv->kv_len) || (kv->n_page_ids && !kv->page_ids)) return PTC_ERR_INVALID_ARG;
  if (kv->n_pages && (!aligned16(kv->k) || !aligned16(kv->v))) return PTC_ERR_INVALID_ARG;
  if (kv->n_req == PTC_NONE || kv->n_pages == PTC_NONE) return PTC_ERR_OVERFLOW;
  const uint32_t ext[3] = {kv->n_pages, kv->n_kv_heads, kv->block_size};
  for (int i = 0; i < 3; ++i)
    if (!stride_ok(kv->k_stride[i], ext[i]) || !stride_ok(kv->v_stride[i], ext[i])) return PTC_ERR_INVALID_ARG;
  o->k = static_cast<char*>(kv->k);
  o->v = static_cast<char*>(kv->v);
  o->ks_page = stride_of(kv->k_stride[0], ext[0]);
  o->ks_head = stride_of(kv->k_stride[1], ext[1]);
  o->ks_slot = stride_of(kv->k_stride[2], ext[2]);
  o->vs_page = stride_of(kv->v_stride[0], ext[0]);
  o->vs_head = stride_of(kv->v_stride[1], ext[1]);
  o->vs_slot = stride_of(kv->v_stride[2], ext[2]);
  o->page_ids = kv->page_ids;
  o->page_off = kv->page_off;
  o->kv_len = kv->kv_len;
  o->n_page_ids = kv->n_page_ids;
  o->n_pages = kv->n_pages;
  o->n_req = kv->n_req;
  o->B = kv->block_size;
  o->H = kv->n_kv_heads;
  o->D = kv->head_dim;
  return PTC_OK;
}

// The status word of a call: the caller's, or one at the start of the
// workspace, which is cleared here and read by kv_end.
inline ptc_status kv_begin(uint32_t* status, void* ws, cudaStream_t s, uint32_t** word) {
  *word = status ? status : static_cast<uint32_t*>(ws);
  return status ? PTC_OK : fill_async(ws, 0u, 16, s);
}

inline ptc_status kv_end(uint32_t* status, const uint32_t* word, cudaStream_t s) {
  if (cudaGetLastError() != cudaSuccess) return PTC_ERR_CUDA;
  if (status) return PTC_OK;
  uint64_t* pin = host_stage()->out;
  if (copy_to_host_async(pin, word, 16, s) != PTC_OK) return PTC_ERR_CUDA;
  if (cudaStreamSynchronize(s) != cudaSuccess) return PTC_ERR_CUDA;
  timer_resolve();
  return static_cast<ptc_status>(*reinterpret_cast<const uint32_t*>(pin));
}

// Lets a kernel have `bytes` of dynamic shared memory, once on every device.
template <typename F>
bool large_smem(F* kernel, int bytes, std::atomic<uint64_t>& ready) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (ready.load(std::memory_order_relaxed) & bit) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  ready.fetch_or(bit, std::memory_order_relaxed);
  return true;
}

constexpr size_t kKvStatusBytes = 256;

}  // namespace ptc
