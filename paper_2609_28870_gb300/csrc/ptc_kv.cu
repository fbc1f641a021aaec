// Paged keys and values: the write of new tokens (ptc_kv_append) and the
// eviction by accumulated attention weight (ptc_kv_evict).
#include "ptc_kv.cuh"

namespace ptc {
namespace {

// ------------------------------------------------------------------ append
// A copy: T rows of H * D values for k and for v, read and written once, so
// HBM bounds it.  A CTA takes `per` consecutive tokens; one thread a token
// finds the token's request and slot, then all threads move 16 bytes each.
// 34,692 tokens of 8 heads of 128, 0.28 GB: 48 us, 5.9 TB/s; 64 tokens 3.8 us,
// launch and three dependent reads.
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
__host__ __device__ __forceinline__ uint32_t div_up(uint32_t a, uint32_t b) { return (a + b - 1) / b; }

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
  uint32_t* status;
};

// Whether request r's lists are sound and the destination has room for its b tokens.
__device__ __forceinline__ bool evict_ok(const EvictArgs& a, uint32_t r, uint32_t n, uint32_t b) {
  const uint64_t d0 = a.dst_off[r], d1 = a.dst_off[r + 1];
  return pages_hold(a.kv, r, n) && n <= a.max_kv_len && d0 <= d1 && d1 <= a.n_dst_ids && b <= (d1 - d0) * a.kv.B;
}

// Weights as integers in the same order: NaN lowest (1), -0 equal to 0, and
// +infinity below kForced, which stands for tokens that are kept in any case;
// 0 stands for no token.
constexpr uint32_t kForced = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 1u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The kept tokens of a request and key head: the weight that the need-th
// heaviest of [n_sink, n - n_recent) has, by a radix search over 11, 11 and 10
// bits of the ordered weights, then the positions above it, and the first of
// those equal to it, in order.  Reading the weights is a few microseconds, so the
// time is the chain of passes over one request's tokens: a cluster of CTAs
// takes them, each a slice that it reads once and keeps in shared memory (or
// reads again in every pass, where a slice is longer than that), and adds its
// histogram and its counts up with the others' through their shared memory.
// 131,072 tokens by 8 CTAs take 25 us, 12 requests of 9K to 131K with 8 heads
// 58 us (one CTA a head: 369 us), in 2.5 waves: the longest request sizes the
// clusters of all.
constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;
constexpr uint32_t kSelBins = 2048;
constexpr uint32_t kSelSlice = 40960;     // tokens of a slice that shared memory holds
constexpr uint32_t kSelMaxCluster = 8;

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t ld_cluster(const uint32_t* p, uint32_t rank) {
  uint32_t at, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

// Inclusive sums along the warp.
__device__ __forceinline__ uint32_t scan_warp(uint32_t x) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(kFull, x, o);
    if ((threadIdx.x & 31) >= (uint32_t)o) x += y;
  }
  return x;
}

struct SelShared {
  uint32_t hist[2][kSelBins];  // of even and odd passes
  uint32_t coarse[2][64];      // sums of 32 bins
  uint32_t warp[kSelWarps], ties[kSelWarps];
  uint32_t bin, above, in_bin;
  uint32_t count[2];           // of the slice: kept above the threshold, equal to it
};

__global__ void __launch_bounds__(kSelThreads, 2) k_evict_select(const EvictArgs a, uint32_t clusters, uint32_t slice_cap) {
  grid_dep_sync();
  extern __shared__ __align__(16) float s_w[];  // slice_cap of them, or none
  __shared__ SelShared sh;
  const uint32_t rank = blockIdx.x % clusters, h = blockIdx.x / clusters, r = blockIdx.y;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t n = a.kv.kv_len[r], b = n < a.n_keep ? n : a.n_keep;
  const uint64_t d0 = a.dst_off[r], d1 = a.dst_off[r + 1];
  const bool ok = evict_ok(a, r, n, b);
  if (h == 0 && rank == 0 && tid == 0) {
    a.new_len[r] = b;
    if (!ok) report(a.status, PTC_ERR_INVALID_ARG);
  }
  if (r == 0) {  // slots of no request
    const uint64_t lo = a.dst_off[0] * a.kv.B, hi = a.dst_off[a.kv.n_req] * a.kv.B, end = a.n_dst_ids * a.kv.B;
    if (lo <= hi && hi <= end)
      for (uint64_t i = rank * kSelThreads + tid; i < lo + (end - hi); i += clusters * kSelThreads)
        a.new_mass[h * a.new_mass_stride + (i < lo ? i : hi + i - lo)] = 0.f;
  }
  if (!ok) return;  // the whole cluster
  uint32_t* keep = a.keep + ((uint64_t)r * a.kv.H + h) * a.n_keep;
  const float* w = a.mass + h * a.mass_stride + a.kv.page_off[r] * a.kv.B;
  float* new_w = a.new_mass + h * a.new_mass_stride + d0 * a.kv.B;
  const uint32_t all = clusters * kSelThreads, me = rank * kSelThreads + tid;
  for (uint32_t i = b + me; i < a.n_keep; i += all) keep[i] = kNone;
  for (uint64_t i = b + me; i < (d1 - d0) * a.kv.B; i += all) new_w[i] = 0.f;
  if (b == n) {
    for (uint32_t i = me; i < n; i += all) {
      keep[i] = i;
      new_w[i] = w[i];
    }
    return;
  }
  // the slice: a whole number of 128 tokens a warp
  const uint32_t per_warp = (div_up(n, clusters * kSelWarps) + 127) & ~127u, slice = per_warp * kSelWarps;
  const uint32_t s0 = rank * slice;
  const uint32_t lo = a.n_sink, hi = n - a.n_recent;
  const bool held = slice <= slice_cap;
  if (held) {
    // eight loads in flight a thread (past the end: the last token's weight, not used)
    for (uint32_t j0 = tid; j0 < slice; j0 += 8 * kSelThreads) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint32_t j = s0 + j0 + u * kSelThreads;
        x[u] = __ldg(w + (j < n ? j : n - 1));
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (j0 + u * kSelThreads < slice) s_w[j0 + u * kSelThreads] = x[u];
    }
    __syncthreads();
  }
  // four tokens of the slice
  auto weights_of = [&](uint32_t j) {
    if (held) return *reinterpret_cast<const float4*>(s_w + j);
    auto one = [&](uint32_t x) { return __ldg(w + (s0 + x < n ? s0 + x : n - 1)); };
    return make_float4(one(j), one(j + 1), one(j + 2), one(j + 3));
  };
  auto keys_of = [&](uint32_t j, const float4& x) {
    uint4 k = make_uint4(order_of(x.x), order_of(x.y), order_of(x.z), order_of(x.w));
    const uint32_t at = s0 + j;
    if (at < lo || at + 4 > hi) {
      auto one = [&](uint32_t y, uint32_t key) { return y >= n ? 0u : y < lo || y >= hi ? kForced : key; };
      k = make_uint4(one(at, k.x), one(at + 1, k.y), one(at + 2, k.z), one(at + 3, k.w));
    }
    return k;
  };
  uint32_t need = b - a.n_sink - a.n_recent;
  // prefix holds the bits of the threshold settled so far
  uint32_t prefix = 0, mask = 0;
  bool whole_bin = false;
  if (need) {
#pragma unroll 1
    for (int pass = 0; pass < 3 && !whole_bin; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t bins = pass == 2 ? 1024 : 2048;
      uint32_t* hist = sh.hist[pass & 1];
      for (uint32_t i = tid; i < kSelBins; i += kSelThreads) hist[i] = 0;
      __syncthreads();
#pragma unroll 2
      for (uint32_t j = 4 * tid; j < slice; j += 4 * kSelThreads) {
        const uint4 v = keys_of(j, weights_of(j));
        const uint32_t k[4] = {v.x, v.y, v.z, v.w};
        // a run of equal weights counts at once
        const uint32_t b0 = (v.x >> shift) & (bins - 1);
        const bool in0 = (v.x & mask) == prefix;
        if (v.x == v.y && v.x == v.z && v.x == v.w) {
          if (in0) atomicAdd(&hist[b0], 4u);
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if ((k[x] & mask) == prefix) atomicAdd(&hist[(k[x] >> shift) & (bins - 1)], 1u);
        }
      }
      __syncthreads();
      // sums of 32 bins; then one warp looks for the bin, first among the
      // cluster's sums, then among the 32 bins
#pragma unroll
      for (uint32_t x = warp * (64 / kSelWarps); x < (warp + 1) * (64 / kSelWarps); ++x) {
        // bins of kForced in the first pass: weights end below
        const uint32_t at = 32 * x + lane, all_of = __reduce_add_sync(kFull, pass == 0 && at > 2044 ? 0u : hist[at]);
        if (lane == 0) sh.coarse[pass & 1][x] = all_of;
      }
      cluster_sync_all();
      if (warp == 0) {
        uint32_t c[2] = {0, 0};  // sums 63 - 2 lane and 62 - 2 lane
#pragma unroll
        for (uint32_t x = 0; x < kSelMaxCluster; ++x) {
          if (x >= clusters) break;
          c[0] += ld_cluster(&sh.coarse[pass & 1][63 - 2 * lane], x);
          c[1] += ld_cluster(&sh.coarse[pass & 1][62 - 2 * lane], x);
        }
        uint32_t before = scan_warp(c[0] + c[1]) - c[0] - c[1];
        // the first sum, from the top, that reaches `need`
        const bool one = before < need && need <= before + c[0];
        const bool two = before + c[0] < need && need <= before + c[0] + c[1];
        const int src = __ffs(__ballot_sync(kFull, one || two)) - 1;
        const uint32_t at = __shfl_sync(kFull, one ? 63 - 2 * lane : 62 - 2 * lane, src);
        const uint32_t up = __shfl_sync(kFull, one ? before : before + c[0], src);
        const uint32_t mine = 32 * at + 31 - lane;  // of the 32 bins, from the top
        uint32_t k = 0;
#pragma unroll
        for (uint32_t x = 0; x < kSelMaxCluster; ++x) {
          if (x >= clusters) break;
          k += ld_cluster(hist + mine, x);
        }
        if (pass == 0 && mine > 2044) k = 0;
        before = up + scan_warp(k) - k;
        if (before < need && need <= before + k) {
          sh.bin = mine;
          sh.above = before;
          sh.in_bin = k;
        }
      }
      __syncthreads();
      prefix |= sh.bin << shift;
      mask |= (bins - 1) << shift;
      need -= sh.above;
      whole_bin = need == sh.in_bin;  // all of the bin is kept: what is left of the bits does not matter
      __syncthreads();
    }
  } else {
    prefix = kForced - 1;  // above every weight
    mask = 0xFFFFFFFFu;
  }
  // a warp's stretch of the slice: how many are above the threshold (or kept
  // in any case), how many equal to it; then where they go.  Both counts in one
  // word, 16 bits each (a lane's four tokens, a warp's 128).
  const uint32_t t0 = warp * per_warp, t1 = t0 + per_warp;
  auto look = [&](uint32_t j, const float4& x) {
    const uint4 v = keys_of(j + 4 * lane, x);
    const uint32_t k[4] = {v.x & mask, v.y & mask, v.z & mask, v.w & mask};
    uint32_t bits = 0;  // above: bits 0-3, equal: bits 16-19
#pragma unroll
    for (int x = 0; x < 4; ++x) bits |= (k[x] > prefix ? 1u << x : 0u) | (k[x] == prefix ? 0x10000u << x : 0u);
    return bits;
  };
  uint32_t n_up = 0, n_eq = 0;
  for (uint32_t j = t0; j < t1; j += 128) {
    const uint32_t bits = look(j, weights_of(j + 4 * lane));
    n_up += __popc(bits & 0xFFFFu);
    n_eq += __popc(bits >> 16);
  }
  n_up = __reduce_add_sync(kFull, n_up);
  n_eq = __reduce_add_sync(kFull, n_eq);
  if (lane == 0) {
    sh.warp[warp] = n_up;
    sh.ties[warp] = n_eq;
  }
  __syncthreads();
  uint32_t up_at = 0, eq_at = 0;
  for (uint32_t x = 0; x < warp; ++x) {
    up_at += sh.warp[x];
    eq_at += sh.ties[x];
  }
  if (tid == kSelThreads - 1) {
    sh.count[0] = up_at + n_up;
    sh.count[1] = eq_at + n_eq;
  }
  cluster_sync_all();
  for (uint32_t x = 0; x < rank; ++x) {
    up_at += ld_cluster(&sh.count[0], x);
    eq_at += ld_cluster(&sh.count[1], x);
  }
  if (n_up || n_eq)
    for (uint32_t j = t0; j < t1; j += 128) {
      const float4 x4 = weights_of(j + 4 * lane);
      const float raw[4] = {x4.x, x4.y, x4.z, x4.w};
      const uint32_t bits = look(j, x4);
      const uint32_t mine = __popc(bits & 0xFFFFu) | __popc(bits >> 16) << 16;
      uint32_t incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(kFull, incl, o);
        if (lane >= (uint32_t)o) incl += y;
      }
      const uint32_t before = incl - mine;
      uint32_t up = up_at + (before & 0xFFFFu), eq = eq_at + (before >> 16);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool above = bits >> x & 1, equal = bits >> (16 + x) & 1;
        if (above || (equal && eq < need)) {
          const uint32_t at = up + (eq < need ? eq : need), from = s0 + j + 4 * lane + x;
          keep[at] = from;
          new_w[at] = raw[x];
        }
        up += above;
        eq += equal;
      }
      const uint32_t total = __shfl_sync(kFull, incl, 31);
      up_at += total & 0xFFFFu;
      eq_at += total >> 16;
    }
  cluster_sync_all();  // no CTA ends while another reads its counts
}

constexpr int kMvThreads = 256;
constexpr uint32_t kMvRows = 32;

// The move: kMvRows kept rows of one request and head a CTA.  HBM bounds it:
// 96 times 8,192 rows of k and v, 0.81 GB read and written, 122 us, 6.6 TB/s.
// (In one kernel with the selection, behind each cluster's own, the rows of few
// heads at a time were in flight: 271 us for both against 180.)
__global__ void __launch_bounds__(kMvThreads) k_evict_move(EvictArgs a) {
  grid_dep_sync();
  const uint32_t h = blockIdx.y, r = blockIdx.z, i0 = blockIdx.x * kMvRows;
  const uint32_t n = a.kv.kv_len[r], b = n < a.n_keep ? n : a.n_keep;
  if (i0 >= b || !evict_ok(a, r, n, b)) return;
  const uint64_t p0 = a.kv.page_off[r], d0 = a.dst_off[r];
  const uint32_t* keep = a.keep + ((uint64_t)r * a.kv.H + h) * a.n_keep;
  const uint32_t rows = b - i0 < kMvRows ? b - i0 : kMvRows, chunks = a.kv.D / 8;
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
  }
}

// CTAs a request and head: enough that a slice is at most 4,096 tokens (the
// passes over a slice are then as short as the exchanges between them), as long
// as all of them are on the GPU at once (two an SM), and at any rate so many
// that a slice is at most 10,240, if 8 are.
void launch_select(const EvictArgs& a, cudaStream_t s) {
  const uint64_t pairs = (uint64_t)a.kv.H * a.kv.n_req, room = 2 * (uint64_t)num_sms();
  uint32_t c = 1;
  auto slice = [&](uint32_t x) { return div_up(a.max_kv_len, x); };
  while (c < kSelMaxCluster && ((slice(c) > 4096 && 2 * c * pairs <= room) || slice(c) > kSelSlice / 4)) c *= 2;
  // slices are rounded up to 128 tokens a warp
  const uint32_t cap = slice(c) + 2048 <= kSelSlice ? slice(c) + 2048 : 0, smem = cap * 4;
  static std::atomic<uint64_t> ready{0};
  (void)large_smem(k_evict_select, kSelSlice * 4, ready);  // a failure shows at the launch
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = c;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.kv.H * c, a.kv.n_req);
  cfg.blockDim = kSelThreads;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, k_evict_select, a, c, cap);
}


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
  if (!status && !ws_ok(ws, ws_bytes, kKvStatusBytes)) return PTC_ERR_WORKSPACE;
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

extern "C" size_t ptc_kv_evict_workspace_bytes(uint32_t, uint32_t, uint32_t) { return kKvStatusBytes; }

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
  if (!status && !ws_ok(ws, ws_bytes, kKvStatusBytes)) return PTC_ERR_WORKSPACE;
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
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  PTC_LAUNCH("k_evict_select", s, launch_select(a, s));
  const uint32_t most = n_keep < max_kv_len ? n_keep : max_kv_len;
  const uint32_t gx = most ? (most + kMvRows - 1) / kMvRows : 1;
  PTC_KERNEL("k_evict_move", s, k_evict_move, dim3(gx, kv->n_kv_heads, kv->n_req), kMvThreads, 0, a);
  return kv_end(status, a.status, s);
}
