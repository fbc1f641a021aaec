// Attention of new tokens over paged keys and values (ptc_paged_attention).
#include <cmath>

#include "ptc_attn_tiles.cuh"

namespace ptc {
namespace {

// req_search over offsets that this kernel has written itself.
__device__ __forceinline__ uint32_t unit_search(const uint64_t* off, uint32_t lo, uint32_t hi, uint64_t u) {
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    if (ld_relaxed_u64(off + mid) <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The requests' share of the units, and every CTA's start, for the tiles
// (blockIdx.y = 0) or the weights (1).  The time of a call of few units is a
// chain of latencies: what the lists hold is read once and kept in shared
// memory (the first kPlanThreads requests of it), and the CTAs here add it up
// each for itself and find 32 starts each, one a warp (one CTA for all starts
// took 10 us, of which 8 were spent on them).
constexpr int kPlanThreads = 1024;
__global__ void __launch_bounds__(kPlanThreads) k_attn_plan(AttnArgs a) {
  asm volatile("griddepcontrol.launch_dependents;");
  grid_dep_sync();
  __shared__ uint64_t s_warp[32], s_off[kPlanThreads + 1];
  __shared__ uint32_t s_m[kPlanThreads], s_n[kPlanThreads];
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, R = a.kv.n_req, tq = a.tq;
  const bool weights = blockIdx.y == 1;
  const uint32_t span = 2 * tq, ctas = a.ctas;
  auto extra_of = [&](uint32_t m, uint32_t i) { return weights ? kMassExtra : tile_extra(m, span, a.tq32, i); };
  AttnPlan* plan = a.plan + blockIdx.y;
  uint64_t* unit_off = a.unit_off + (uint64_t)blockIdx.y * (R + 1);
  // a request's first-level tiles, and the units of one of them
  auto tiles_of = [&](uint32_t m, uint32_t n) { return weights ? (m ? div_up(n, kMassKeys) : 0u) : div_up(m, span); };
  auto units_of = [&](uint32_t m, uint32_t n, uint32_t i) {
    return extra_of(m, i) + (weights ? div_up(m, tq) - first_seeing(m, n, tq, i) : key_tiles(m, n, span, i));
  };
  bool bad = tid == 0 && (a.tok_off[0] != 0 || a.tok_off[R] != a.n_tok);
  uint64_t carry = 0;
  if (blockIdx.x == 0 && tid < kMaxCtas) plan->arrived[tid] = 0;
  for (uint32_t r0 = 0; r0 < R; r0 += kPlanThreads) {
    const uint32_t r = r0 + tid;
    uint32_t m = 0, n = 0;
    if (r < R) {
      const uint64_t lo = a.tok_off[r], hi = a.tok_off[r + 1];
      n = a.kv.kv_len[r];
      const bool hold = pages_hold(a.kv, r, n);
      const bool wrong = (lo > hi) | (hi > a.n_tok) | (hi - lo > a.max_q_len) | (n > a.most) | !hold;
      bad |= wrong;
      m = wrong ? 0 : (uint32_t)(hi - lo);
    }
    const uint32_t tiles = tiles_of(m, n);
    uint64_t mine = 0;
    if (tiles <= 2)
      for (uint32_t i = 0; i < tiles; ++i) mine += units_of(m, n, i);
    // requests of many tiles: a warp adds one up
    for (uint32_t todo = __ballot_sync(kFull, tiles > 2); todo; todo &= todo - 1) {
      const int src = __ffs(todo) - 1;
      const uint32_t mm = __shfl_sync(kFull, m, src), nn = __shfl_sync(kFull, n, src),
                     tt = __shfl_sync(kFull, tiles, src);
      uint64_t sum = 0;
      for (uint32_t i = lane; i < tt; i += 32) sum += units_of(mm, nn, i);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
      if (lane == (uint32_t)src) mine = sum;
    }
    mine *= a.kv.H;
    uint64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(kFull, incl, o);
      if (lane >= (uint32_t)o) incl += y;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    uint64_t sums = s_warp[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(kFull, sums, o);
      if (lane >= (uint32_t)o) sums += y;
    }
    const uint64_t earlier = __shfl_sync(kFull, sums, warp ? warp - 1 : 0);
    const uint64_t before = carry + incl - mine + (warp ? earlier : 0), all = carry + __shfl_sync(kFull, sums, 31);
    if (r < R) unit_off[r] = before;
    if (r0 == 0) {
      s_off[tid] = before;
      s_m[tid] = m;
      s_n[tid] = n;
    }
    carry = all;
    __syncthreads();
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    unit_off[R] = carry;
    if (blockIdx.x == 0) plan->ok = !bad;
    if (bad) report(a.status, PTC_ERR_INVALID_ARG);
  }
  if (bad) return;
  const bool shared = R <= kPlanThreads;
  if (tid == 0 && shared) s_off[R] = carry;
  __syncthreads();
  // 64-bit divisions are long; hardly a call needs one
  auto ratio = [](uint64_t x, uint64_t y) { return x >> 32 || y >> 32 ? x / y : (uint64_t)((uint32_t)x / (uint32_t)y); };
  const uint64_t each = ratio(carry, ctas);
  const uint32_t over = (uint32_t)(carry - each * ctas);
  const uint32_t c = blockIdx.x * 32 + warp;
  if (c <= ctas) {
    CtaStart s{};
    s.u = each * c + over * c / ctas;
    uint32_t m = 0, n = 0;
    if (s.u < carry) {
      uint64_t from, to;
      if (shared) {
        uint32_t lo = 0, hi = R - 1;
        while (lo < hi) {
          const uint32_t mid = lo + (hi - lo + 1) / 2;
          if (s_off[mid] <= s.u) lo = mid;
          else hi = mid - 1;
        }
        s.r = lo;
        m = s_m[lo];
        n = s_n[lo];
        from = s_off[lo];
        to = s_off[lo + 1];
      } else {
        s.r = unit_search(unit_off, 0, R - 1, s.u);
        m = (uint32_t)(a.tok_off[s.r + 1] - a.tok_off[s.r]);
        n = a.kv.kv_len[s.r];
        from = ld_relaxed_u64(unit_off + s.r);
        to = ld_relaxed_u64(unit_off + s.r + 1);
      }
      const uint64_t head = ratio(to - from, a.kv.H), in = s.u - from;
      s.h = (uint32_t)ratio(in, head);
      uint64_t rest = in - s.h * head;
      const uint32_t tiles = tiles_of(m, n);
      for (uint32_t t0 = 0; t0 < tiles; t0 += 32) {
        const uint32_t k = t0 + lane < tiles ? units_of(m, n, t0 + lane) : 0;
        uint32_t incl = k;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(kFull, incl, o);
          if (lane >= (uint32_t)o) incl += y;
        }
        const uint32_t here = __ballot_sync(kFull, rest < incl);
        if (here) {
          const int src = __ffs(here) - 1;
          s.major = t0 + src;
          const uint32_t at = (uint32_t)rest - __shfl_sync(kFull, incl - k, src), extra = extra_of(m, s.major);
          s.minor = at > extra ? at - extra : 0;
          const uint32_t all = __shfl_sync(kFull, k, src) - extra;
          const uint32_t least = weights || m - s.major * span <= a.tq32 ? 1 : kPartMin;
          if (s.minor < least) {
            s.u -= at;
            s.minor = 0;
          } else if (all - s.minor < least) {
            s.u += extra + all - at;
            s.minor = all;
          }
          break;
        }
        rest -= __shfl_sync(kFull, incl, 31);
      }
    }
    if (s.u < carry) {
      s.m = m;
      s.n = n;
      s.tok0 = a.tok_off[s.r];
      s.page0 = a.kv.page_off[s.r];
    }
    if (lane == 0) plan->start[c] = s;
  }
}

// cuTensorMapEncodeTiled, from the driver that the runtime has loaded.
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return static_cast<EncodeFn>(nullptr);
    }
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

bool encode(CUtensorMap* map, bool bf16, void* base, const cuuint64_t (&dims)[4], const cuuint64_t (&strides)[3],
            const cuuint32_t (&boxes)[4]) {
  const cuuint32_t steps[4] = {1, 1, 1, 1};
  const EncodeFn fn = encoder();
  return fn && fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, strides,
                  boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

void launch_plan(const AttnArgs& a, bool weights, cudaStream_t s) {
  PTC_KERNEL("k_attn_plan", s, k_attn_plan, dim3(a.ctas / 32 + 1, weights ? 2 : 1), kPlanThreads, 0, a);
}

namespace {

template <typename T, int NSLAB, bool TMA, int KIND>
ptc_status launch_one(const AttnArgs& a, const CUtensorMap (&m)[4], cudaStream_t s) {
  constexpr int smem = TileShape<NSLAB, KIND>::kSmem;
  static std::atomic<uint64_t> ready{0};
  const auto kernel = k_attn_tiles<T, NSLAB, TMA, KIND>;
  if (!large_smem(kernel, smem, ready)) return PTC_ERR_CUDA;
  PTC_KERNEL("k_attn_tiles", s, kernel, a.ctas, kTileThreads, smem, m[0], m[1], m[2], m[3], a);
  return PTC_OK;
}
template <typename T, int NSLAB>
ptc_status launch_tiles(const AttnArgs& a, const CUtensorMap (&m)[4], bool tma, cudaStream_t s) {
  if (a.max_q_len <= a.tq32) return tma ? launch_one<T, NSLAB, true, kFew>(a, m, s) : launch_one<T, NSLAB, false, kFew>(a, m, s);
  return tma ? launch_one<T, NSLAB, true, kAny>(a, m, s) : launch_one<T, NSLAB, false, kAny>(a, m, s);
}

template <typename T>
ptc_status launch(AttnArgs& a, cudaStream_t s) {
  constexpr bool bf16 = Weights<T>::kBf16;
  const bool by_tiles = a.mass_out && !a.scores && a.n_tok;  // the weights' own tiles
  // copies of whole groups of 8 rows that neither leave a page nor a tile
  a.box = kKeys;
  while (a.kv.B % a.box) a.box /= 2;
  const bool tma = a.n_tok && a.box >= 8 && a.kv.n_pages > 0;
  launch_plan(a, by_tiles, s);
  CUtensorMap m[4] = {};
  if (a.n_tok) {
    if (tma && (!cache_map(&m[0], a.kv, bf16, a.kv.k, a.kv.ks_page, a.kv.ks_head, a.kv.ks_slot, a.box) ||
                !cache_map(&m[1], a.kv, bf16, a.kv.v, a.kv.vs_page, a.kv.vs_head, a.kv.vs_slot, a.box)))
      return PTC_ERR_CUDA;
    if (!tokens_map(&m[2], a, bf16, a.tq) || (a.tq32 && !tokens_map(&m[3], a, bf16, a.tq32))) return PTC_ERR_CUDA;
    const ptc_status st = a.kv.D > 64 ? launch_tiles<T, 2>(a, m, tma, s) : launch_tiles<T, 1>(a, m, tma, s);
    if (st != PTC_OK) return st;
  }
  return a.mass_out && a.kv.n_page_ids ? launch_mass(a, bf16, m[0], m[2], tma, s) : PTC_OK;
}

// Scores kept for the weights: none without them or where requests have more rows.
uint64_t kept_scores(uint32_t n_q_heads, uint32_t n_kv_heads, uint32_t max_q_len, uint64_t mass_stride) {
  const uint64_t rows = (uint64_t)max_q_len * (n_kv_heads ? n_q_heads / n_kv_heads : 0);
  return rows <= kFewRows ? rows * n_kv_heads * mass_stride : 0;
}

}  // namespace

ptc_status launch_attention(AttnArgs& a, bool bf16, cudaStream_t s) {
  return bf16 ? launch<__nv_bfloat16>(a, s) : launch<__half>(a, s);
}

AttnWs attn_ws(uint32_t n_req, uint32_t ctas, uint32_t D, uint64_t scores) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  AttnWs w;
  w.plan = kKvStatusBytes;
  w.units = w.plan + up(2 * sizeof(AttnPlan));
  w.ml = w.units + up(2 * (size_t)(n_req + 1) * 8);
  w.part = w.ml + up((size_t)2 * ctas * kRows * 8);
  w.mass = w.part + up((size_t)2 * ctas * kRows * D * 4);
  w.scores = w.mass + up((size_t)2 * ctas * kMassKeys * 4);
  w.total = w.scores + up(scores * 4);
  return w;
}
uint32_t tile_ctas() {
  static const uint32_t n = [] {
    const int x = num_sms();
    return x < (int)kMaxCtas ? (uint32_t)x : kMaxCtas;
  }();
  return n;
}
void attn_place(AttnArgs& a, const AttnWs& at, char* w) {
  a.ctas = tile_ctas();
  a.plan = reinterpret_cast<AttnPlan*>(w + at.plan);
  a.unit_off = reinterpret_cast<uint64_t*>(w + at.units);
  a.part_ml = reinterpret_cast<float2*>(w + at.ml);
  a.part = reinterpret_cast<float*>(w + at.part);
  a.part_mass = reinterpret_cast<float*>(w + at.mass);
}
ptc_status attn_call(AttnArgs& a, const ptc_paged_kv* kv, const uint64_t* tok_off, uint64_t n_tok, const int64_t* q_stride,
                     uint32_t n_q_heads, float scale) {
  if (!tok_off || !q_stride || n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return PTC_ERR_INVALID_ARG;
  if (n_q_heads / kv->n_kv_heads > kMaxGroup) return PTC_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale) || (n_tok && !kv->n_req)) return PTC_ERR_INVALID_ARG;
  if (!std::isfinite(scale * kLog2e)) return PTC_ERR_INVALID_ARG;
  a.tok_off = tok_off;
  a.n_tok = n_tok;
  a.n_q_heads = n_q_heads;
  a.G = n_q_heads / kv->n_kv_heads;
  a.tq = 128 / a.G;
  a.tq32 = 32 / a.G;
  a.scale = scale;
  a.most = 0xFFFFFFFFu;
  return PTC_OK;
}
ptc_status attn_rows(AttnArgs& a, const void* q, const int64_t* q_stride, uint32_t max_q_len, void* out, float* lse) {
  if (a.n_tok && (!aligned16(q) || !aligned16(out) || !lse)) return PTC_ERR_INVALID_ARG;
  const uint32_t ext[2] = {(uint32_t)a.n_tok, a.n_q_heads};
  for (int i = 0; i < 2; ++i)
    if (!stride_ok(q_stride[i], ext[i])) return PTC_ERR_INVALID_ARG;
  a.q = static_cast<const char*>(q);
  a.q_tok = stride_of(q_stride[0], ext[0]);
  a.q_head = stride_of(q_stride[1], ext[1]);
  a.max_q_len = max_q_len;
  a.out = static_cast<char*>(out);
  a.lse = lse;
  const uint32_t wait_test = test_wait_polls(PTC_TEST_WAIT_ATTENTION);
  a.withhold = wait_test != 0;
  a.limit = wait_test ? 1024ll * wait_test : kMbarCycles;
  return PTC_OK;
}

// The cache as [page][head][slot][d], read 64 columns by `box` slots at a time.
bool cache_map(CUtensorMap* map, const KvView& kv, bool bf16, char* base, int64_t page, int64_t head, int64_t slot,
               uint32_t box) {
  const cuuint64_t dims[4] = {kv.D, kv.B, kv.H, kv.n_pages};
  const cuuint64_t strides[3] = {2 * (cuuint64_t)slot, 2 * (cuuint64_t)head, 2 * (cuuint64_t)page};
  const cuuint32_t boxes[4] = {64, box, 1, 1};
  return encode(map, bf16, base, dims, strides, boxes);
}

// The queries as [token][key head][head of the group][d], read 64 columns by
// `tokens` whole tokens of one key head at a time.
bool tokens_map(CUtensorMap* map, const AttnArgs& a, bool bf16, uint32_t tokens) {
  const cuuint64_t dims[4] = {a.kv.D, a.G, a.kv.H, a.n_tok};
  const cuuint64_t strides[3] = {2 * (cuuint64_t)a.q_head, 2 * (cuuint64_t)a.q_head * a.G, 2 * (cuuint64_t)a.q_tok};
  const cuuint32_t boxes[4] = {64, a.G, 1, tokens};
  return encode(map, bf16, const_cast<char*>(a.q), dims, strides, boxes);
}

}  // namespace ptc

using namespace ptc;

extern "C" size_t ptc_paged_attention_workspace_bytes(uint32_t n_req, uint32_t n_q_heads, uint32_t n_kv_heads,
                                                      uint32_t head_dim, uint32_t max_q_len, uint64_t mass_stride) {
  return attn_ws(n_req, tile_ctas(), head_dim, kept_scores(n_q_heads, n_kv_heads, max_q_len, mass_stride)).total;
}

extern "C" ptc_status ptc_paged_attention(const ptc_paged_kv* kv, const void* q, const int64_t q_stride[2],
                                          const uint64_t* tok_off, uint64_t n_tok, uint32_t n_q_heads,
                                          uint32_t max_q_len, float scale, void* out, float* lse,
                                          const float* mass_in, float* mass_out, uint64_t mass_stride, void* ws,
                                          size_t ws_bytes, uint32_t* status, void* stream) {
  AttnArgs a{};
  const ptc_status st = kv_view(kv, &a.kv);
  if (st != PTC_OK) return st;
  const ptc_status fits = attn_call(a, kv, tok_off, n_tok, q_stride, n_q_heads, scale);
  if (fits != PTC_OK) return fits;
  // (a stride of up to 2^40 times the scores' rows, at most kFewRows a key head, stays below 2^64 bytes)
  if (n_tok > 0x7FFFFFFFu || n_tok * n_q_heads > (uint64_t(1) << 31) ||
      kv->n_page_ids > (uint64_t(1) << 38) / kv->block_size || (mass_out && mass_stride > uint64_t(1) << 40))
    return PTC_ERR_OVERFLOW;
  if (mass_out ? mass_stride / kv->block_size < kv->n_page_ids : mass_in != nullptr) return PTC_ERR_INVALID_ARG;
  if (kv->n_pages > 0x7FFFFFFFu) return PTC_ERR_OVERFLOW;  // tensor copies have signed coordinates
  const uint64_t scores = mass_out ? kept_scores(n_q_heads, kv->n_kv_heads, max_q_len, mass_stride) : 0;
  const AttnWs at = attn_ws(kv->n_req, tile_ctas(), kv->head_dim, scores);
  if (!ws_ok(ws, ws_bytes, at.total)) return PTC_ERR_WORKSPACE;
  if (kv->n_req == 0) return PTC_OK;
  const ptc_status rows = attn_rows(a, q, q_stride, max_q_len, out, lse);
  if (rows != PTC_OK) return rows;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  a.mass_in = mass_in;
  a.mass_out = mass_out;
  a.mass_stride = mass_stride;
  char* w = static_cast<char*>(ws);
  attn_place(a, at, w);
  a.scores = scores && n_tok ? reinterpret_cast<float*>(w + at.scores) : nullptr;
  a.few = max_q_len * a.G;
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  const ptc_status run = launch_attention(a, kv->dtype == PTC_DTYPE_BF16, s);
  if (run != PTC_OK) return run;
  return kv_end(status, a.status, s);
}
