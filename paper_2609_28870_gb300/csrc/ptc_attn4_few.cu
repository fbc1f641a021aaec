// Attention over pages of 4 bits for requests of few query rows: single tokens,
// or a few of them.
//
// One pass over the keys and values, which HBM bounds if the instructions keep
// up: 6.6 TB/s are 44 values a cycle and SM, so a value has about three of a
// lane's instructions.  They become 16-bit numbers in the registers where the
// matrix instructions want them, with no way through shared memory in 16 bits
// (which tcgen05's operands need, 2 bytes written and read a value):
//   scores   S^T = K Q^T       16 keys x 8 query rows, mma.sync m16n8k16
//   softmax  running maximum and sum of a query row in 32 bits
//   values   O^T += V^T P^T    16 channels x 8 query rows, 16 keys at a time
// The weights are rounded to the cache's 16 bits, as the instructions want both operands
// alike (their sum is not rounded): at most 2^-8, in fp16 2^-11, of each.
// A word of codes is eight neighbouring channels of a key, even ones in its low
// half, so a shifted and masked word is two channels as K's operand wants them;
// the low (high) halves of two keys' words together are one channel of both, as
// V^T's operand does.  Eight query rows are what an instruction's N asks for; 16 and
// 32 take two and four for the same operand.
//
// A call's units are 128 keys of a request's key head, and `kExtra` for what a
// head's tile costs by itself (1, 2, 3, 4: 85, 84, 84, 85 us for 64 single tokens).
// CTA c of C has the units from U c / C on, so where a cut lies, and which CTAs share
// a tile, is arithmetic that every CTA does for itself from the requests' lengths;
// there is no plan to wait for.  A warp takes 32 keys of every 256 and copies its next
// ones into a ring of its own meanwhile, so no warp waits for another until the
// tile's end, where they put their rows together; of a split tile the last CTA that
// is done does so with the parts.
//
// Bounds.  At 128 channels and up to 8 rows 16 keys are 360 instructions of a warp,
// of which the codes take 230 (shift, mask and multiply-add for two values, the
// products, their loads): 12 single tokens over 32K to 131K, 0.57 GB, take 113 us, 5.0
// TB/s, with 63% of the issue slots and 60% of the ALUs' in use at 1.8 GHz; what is
// left waits for fixed latencies, which four warps a scheduler, 128 registers each, do
// not hide.  (165 us with a warp of its own for the copies and 16 keys at a time; 132
// with a mask and an or in one instruction; 125 with the warps' own copies; 119 with
// places in the cache kept a tile; 115 with both blocks' products side by side.)  Two
// and four instructions an operand: 152 and 219 us, at 8 warps an SM.  64 single tokens
// over 1.1K to 12K 81 us, one over 1,012 9 us, a chain of latencies: a launch that
// clears the counts, lengths, pages, keys, parts.
#include "ptc_attn4.cuh"

namespace ptc {
namespace {

constexpr uint32_t kUnit = 128, kChunk = 32, kWarps = 8, kTeam = 4, kThreads = 32 * kWarps;
constexpr uint32_t kExtra = 2;
struct Few4Args {
  KvView kv;
  const char* q;
  int64_t q_tok, q_head;
  const uint64_t* tok_off;
  uint64_t n_tok;
  uint32_t n_q_heads, G, max_q_len;
  float scale;
  char* out;
  float* lse;
  uint32_t* arrived;  // parts of the split tile that begins in CTA c
  float* part;        // unnormalised rows of split tiles: [2 * ctas][rows][64 or 128]
  float2* part_ml;    // their maxima (in powers of two) and sums
  uint32_t ctas;
  uint32_t div_mul, div_shift;  // key / B
  uint32_t k_page16, v_page16;  // BLOCKS: a page's stride by 16
  uint32_t* status;
};

constexpr float kMove4 = 256.f;  // the maximum moves when a weight passes this
constexpr float kNoTop = -3e38f;  // the maximum of no score: any score's weight passes kMove4 by it

template <typename T>
struct Mma16;
template <>
struct Mma16<__nv_bfloat16> {
  static constexpr float kShift = 0.f, kScale = 1.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  // d = A B + c
  static __device__ __forceinline__ void run(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1, float c0, float c1, float c2, float c3) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
  }
};
// (weights of fp16 caches are scaled by 2^7: small ones would fall among fp16's subnormals)
template <>
struct Mma16<__half> {
  static constexpr float kShift = 7.f, kScale = 128.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 x = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ void run(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1, float c0, float c1, float c2, float c3) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
  }
};
// An 8 x 8 matrix of 16-bit numbers over a warp, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// The warp's number, as one value for the warp: what follows from it is left to the
// uniform unit.
__device__ __forceinline__ uint32_t warp_index() { return __shfl_sync(kFull, threadIdx.x >> 5, 0); }

// NS: rows of 64 or 128 channels.  NT: 8, 16 or 32 query rows.
template <int NS, int NT>
struct Shape {
  static constexpr uint32_t kDim = 64 * NS, kRow = NS == 1 ? 48 : 80, kQRows = 8 * NT;
  static constexpr uint32_t kTensor = kChunk * kRow, kStage = 2 * kTensor;  // a warp's chunk
  static constexpr uint32_t kCtas = NS * NT <= 2 ? 2 : 1;  // of an SM: by their registers
  static constexpr uint32_t kRing = kCtas == 1 ? (NT == 4 ? 3 : 4) : NS == 1 ? 3 : 2;
  static constexpr int kBlocks = NS * NT == 8 ? 1 : 2;     // of 16 keys at a time: by the registers again
  static constexpr uint32_t kORow = kDim + 4;  // 32-bit words of a row on its way to the other warps
  static constexpr uint32_t kRegion = NT * 512 * (4 * NS + 1);  // a warp's rows, as lanes hold them or row by row
  static constexpr uint32_t kQueries = 2 * NS * NT * 512;         // the queries' operand; see take_units
  static constexpr uint32_t kRows0 = kWarps * kRing * kStage, kQueries0 = kRows0 + kTeam * kRegion;
  static constexpr uint32_t kBytes = kQueries0 + kQueries;
  static_assert(kQRows * kORow * 4 <= kRegion, "a warp's rows");
};

struct Shared {
  uint64_t off[257];  // units before a block of requests
  uint64_t tok0[256], page0[256];
  uint32_t m[256], n[256];
  uint64_t warp_sum[8];
  float2 ml[kTeam][kFew4Rows];
  uint32_t last;
};

__device__ __forceinline__ uint32_t tiles_of(uint32_t n) { return n ? (n - 1) / kUnit + 1 : 1; }
__device__ __forceinline__ uint64_t units_of(const Few4Args& a, uint32_t m, uint32_t n) {
  return m ? (uint64_t)a.kv.H * (tiles_of(n) + kExtra) : 0;
}

// A CTA's way through its units: tile by tile, keys [kv0, kv1) times 128 of each.
struct Way {
  uint64_t end, tile0, tok0, page0;  // unit after the CTA's last, the tile's first
  uint32_t r, h, m, n, tiles, kv0, kv1;

  __device__ __forceinline__ void request(const Few4Args& a, const Shared& sh) {
    if (a.kv.n_req <= 256) {
      m = sh.m[r];
      n = sh.n[r];
      tok0 = sh.tok0[r];
      page0 = sh.page0[r];
    } else {
      tok0 = a.tok_off[r];
      m = (uint32_t)(a.tok_off[r + 1] - tok0);
      n = a.kv.kv_len[r];
      page0 = a.kv.page_off[r];
    }
    tiles = tiles_of(n);
  }
  // The CTA's keys of the tile at hand; false if it has none.
  __device__ __forceinline__ bool keys(uint64_t from) {
    const uint64_t first = tile0 + kExtra;
    kv0 = from > first ? (uint32_t)(from - first) : 0;
    kv1 = end <= first ? 0 : end - first < tiles ? (uint32_t)(end - first) : tiles;
    return kv0 < kv1;
  }
  __device__ __forceinline__ bool begin(const Few4Args& a, const Shared& sh, uint64_t all, uint32_t c, uint32_t ctas) {
    const uint64_t u = all * c / ctas;
    end = all * (c + 1) / ctas;
    if (u >= end) return false;
    uint32_t lo = 0, hi = 255;
    while (lo < hi) {
      const uint32_t mid = (lo + hi + 1) / 2;
      if (sh.off[mid] <= u) lo = mid;
      else hi = mid - 1;
    }
    uint64_t off = sh.off[lo];
    r = lo;
    if (a.kv.n_req > 256) {  // a block of requests, 32 at a time
      const uint32_t per = (a.kv.n_req + 255) / 256, lane = threadIdx.x & 31;
      for (uint32_t r0 = lo * per;; r0 += 32) {
        const uint32_t x = r0 + lane;
        uint64_t mine = 0;
        if (x < a.kv.n_req && x < (lo + 1) * per) mine = units_of(a, (uint32_t)(a.tok_off[x + 1] - a.tok_off[x]), a.kv.kv_len[x]);
        uint64_t incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint64_t y = __shfl_up_sync(kFull, incl, o);
          if (lane >= (uint32_t)o) incl += y;
        }
        const uint32_t here = __ballot_sync(kFull, u < off + incl);
        if (here) {
          const int src = __ffs(here) - 1;
          r = r0 + src;
          off += __shfl_sync(kFull, incl - mine, src);
          break;
        }
        off += __shfl_sync(kFull, incl, 31);
        if (r0 + 32 >= (lo + 1) * per) return false;  // (the lists are sound, so this is not reached)
      }
    }
    request(a, sh);
    const uint32_t each = tiles + kExtra;
    h = (uint32_t)((u - off) / each);
    tile0 = off + (uint64_t)h * each;
    return keys(u) || next(a, sh);
  }
  __device__ __forceinline__ bool next(const Few4Args& a, const Shared& sh) {
    tile0 += tiles + kExtra;
    if (tile0 + kExtra >= end) return false;
    if (++h == a.kv.H) {
      h = 0;
      do {
        if (++r >= a.kv.n_req) return false;
        request(a, sh);
      } while (m == 0);
    }
    return keys(0);
  }
};

// What a call's requests have of units, and whether its lists are sound.  By the
// whole CTA; request r is of block r / per.
__device__ __forceinline__ bool add_up(const Few4Args& a, Shared& sh, uint64_t& all) {
  const uint32_t tid = threadIdx.x, lane = tid & 31, R = a.kv.n_req, per = (R + 255) / 256;
  bool bad = tid == 0 && (a.tok_off[0] != 0 || a.tok_off[R] != a.n_tok);
  uint64_t mine = 0, incl = 0;
  if (tid < 256) {
    for (uint32_t r = tid * per; r < (tid + 1) * per && r < R; ++r) {
      const uint64_t lo = a.tok_off[r], hi = a.tok_off[r + 1];
      const uint32_t n = a.kv.kv_len[r];
      const bool wrong = (lo > hi) | (hi > a.n_tok) | (hi - lo > a.max_q_len) | !pages_hold(a.kv, r, n) | (n > kMost4);
      bad |= wrong;
      const uint32_t m = wrong ? 0 : (uint32_t)(hi - lo);
      mine += units_of(a, m, n);
      if (per == 1) {
        sh.tok0[r] = lo;
        sh.page0[r] = a.kv.page_off[r];
        sh.m[r] = m;
        sh.n[r] = n;
      }
    }
    incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(kFull, incl, o);
      if (lane >= (uint32_t)o) incl += y;
    }
    if (lane == 31) sh.warp_sum[tid / 32] = incl;
  }
  bad = __syncthreads_or(bad);
  uint64_t before = 0;
  all = 0;
#pragma unroll
  for (uint32_t x = 0; x < 8; ++x) {
    if (x < tid / 32) before += sh.warp_sum[x];
    all += sh.warp_sum[x];
  }
  if (tid < 256) sh.off[tid] = before + incl - mine;
  if (bad && blockIdx.x == 0 && tid == 0) report(a.status, PTC_ERR_INVALID_ARG);
  __syncthreads();
  return !bad;
}

// A warp's copies, chunk by chunk, a chunk or more ahead of its products: 16 bytes a
// lane (cp.async: a tensor or bulk copy of the 1,280 bytes that a head has in a page
// of 16 takes 90 cycles of the SM's one copy engine, 4.1 TB/s; this took 12 contexts
// of 32K to 131K from 140 to 125 us).  BLOCKS: 16 keys lie in a row in one page, else
// every lane finds a key's row.  The pages of the chunk after are asked for
// meanwhile, as a page list comes from HBM too.  Slots of no token read as zeros.
template <int NS, int NT, bool BLOCKS>
struct Feed {
  using S = Shape<NS, NT>;
  static constexpr uint32_t kPieces = kChunk * S::kRow / 16;  // of keys, and of values
  Way w;
  const char *kb, *vb;  // the key head's rows of page 0
  uint32_t chunk, id[2], slot[2], issued;
  bool more;

  __device__ __forceinline__ void head(const Few4Args& a) {
    kb = a.kv.k + w.h * a.kv.ks_head;
    vb = a.kv.v + w.h * a.kv.vs_head;
  }

  // The chunk at hand's first key, or the lane's.
  __device__ __forceinline__ uint32_t key() const {
    return w.kv0 * kUnit + chunk * kChunk + (BLOCKS ? 0 : threadIdx.x & 31);
  }
  // Its pages, of both blocks of 16 or of the lane's key.
  __device__ __forceinline__ void ask(const Few4Args& a) {
    const uint32_t key = this->key();
    const uint32_t at = a.kv.B == 1 ? key : __umulhi(key, a.div_mul) >> a.div_shift;
    const uint32_t* ids = a.kv.page_ids + w.page0;
    slot[0] = key - at * a.kv.B;
    id[0] = key < w.n ? __ldg(ids + at) : kNone;
    if (BLOCKS) {
      const bool over = slot[0] + 16 == a.kv.B;
      slot[1] = over ? 0 : slot[0] + 16;
      id[1] = key + 16 < w.n ? __ldg(ids + at + (over ? 1 : 0)) : kNone;
    }
  }
  // The warp's first chunk of the part at hand or of a later one.
  __device__ __forceinline__ void find(const Few4Args& a, const Shared& sh) {
    const uint32_t warp = warp_index();
    while (more && chunk >= (w.kv1 - w.kv0) * (kUnit / kChunk)) {
      more = w.next(a, sh);
      chunk = warp;
      head(a);
    }
    if (more) ask(a);
  }
  __device__ __forceinline__ void begin(const Few4Args& a, const Shared& sh, const Way& start, bool some) {
    w = start;
    head(a);
    more = some;
    chunk = warp_index();
    issued = 0;
    find(a, sh);
  }
  // Copies the chunk at hand to its place; a group of copies in any case.
  __device__ __forceinline__ void issue(const Few4Args& a, const Shared& sh, uint32_t ring) {
    if (more) {
      const uint32_t lane = threadIdx.x & 31, dst = ring + issued % S::kRing * S::kStage + 16 * lane;
      const uint32_t key = this->key();
      ++issued;
      bool on[2];
      const char *k[2], *v[2];
#pragma unroll
      for (int x = 0; x < (BLOCKS ? 2 : 1); ++x) {
        on[x] = id[x] < a.kv.n_pages;
        if (!on[x] && key + 16 * x < w.n) report(a.status, PTC_ERR_INVALID_ARG);  // (any id: a list may hold kNone)
        if (!on[x]) id[x] = slot[x] = 0;
        if (BLOCKS) {
          const uint32_t in = slot[x] * (S::kRow / 16);
          k[x] = kb + 16 * (uint64_t)(id[x] * a.k_page16 + in);
          v[x] = vb + 16 * (uint64_t)(id[x] * a.v_page16 + in);
        } else {
          k[x] = kb + id[x] * a.kv.ks_page + slot[x] * a.kv.ks_slot;
          v[x] = vb + id[x] * a.kv.vs_page + slot[x] * a.kv.vs_slot;
        }
      }
      if (BLOCKS) {
#pragma unroll
        for (uint32_t i = 0; i < kPieces / 32; ++i) {
          const uint32_t p = lane + 32 * i;
          const bool up = p >= kPieces / 2;
          const uint32_t off = 16 * (up ? p - kPieces / 2 : p);
          cp_async16(dst + 512 * i, (up ? k[1] : k[0]) + off, up ? on[1] : on[0]);
          cp_async16(dst + S::kTensor + 512 * i, (up ? v[1] : v[0]) + off, up ? on[1] : on[0]);
        }
      } else {
        const uint32_t rows = __ballot_sync(kFull, on[0]);
#pragma unroll
        for (uint32_t i = 0; i < kPieces / 32; ++i) {
          const uint32_t p = lane + 32 * i, row = p / (S::kRow / 16), off = 16 * (p % (S::kRow / 16));
          const char* ks = reinterpret_cast<const char*>(__shfl_sync(kFull, reinterpret_cast<uint64_t>(k[0]), row));
          const char* vs = reinterpret_cast<const char*>(__shfl_sync(kFull, reinterpret_cast<uint64_t>(v[0]), row));
          const bool in = rows >> row & 1;
          cp_async16(dst + 512 * i, ks + off, in);
          cp_async16(dst + S::kTensor + 512 * i, vs + off, in);
        }
      }
      chunk += kWarps;
      find(a, sh);
    }
    cp_async_commit();
  }
};

__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
// NS * 2 words.
template <int NS>
__device__ __forceinline__ void lds_words(uint32_t (&x)[2 * NS], uint32_t at) {
  if constexpr (NS == 2)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
  else
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(at) : "memory");
}
template <int NS>
__device__ __forceinline__ void lds_half(uint32_t (&x)[NS], uint32_t at) {
  if constexpr (NS == 2)
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(at) : "memory");
  else
    x[0] = lds32(at);
}

// A warp's rows so far: of query rows 8 i + 2 t and 8 i + 2 t + 1 (t = lane % 4), the
// maximum (as a power of two), the lane's share of the sum, and channels.
template <int NS, int NT>
struct Rows {
  float top[NT][2], l[NT][2], o[NT][4 * NS][4];
};

// Up to 32 keys of a unit, as blocks of 16.  Row i of a block's matrices is key (2 (i %
// 8 / 2) + 4 (i % 2)) % 8 + 8 (i % 2) + i / 8: rows of 80 (48) bytes in that order meet
// no bank twice, neither where four lanes read K's rows whole nor where eight read a
// piece of V's each.
template <typename T, int NS, int NT, int U>
__device__ __forceinline__ void take_keys(uint32_t at, uint32_t key0, uint32_t n, const int32_t (&see)[NT][2], int32_t least,
                                          float sl2, uint32_t q_at, Rows<NS, NT>& st) {
  using S = Shape<NS, NT>;
  using M = Mma16<T>;
  const uint32_t lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  // scores
  const uint32_t kg = ((g & 6) + 4 * (g & 1) & 7) + 8 * (g & 1), group = NS == 2 ? t : t >> 1;
  float s[U][NT][4];
  uint32_t wa[U][2 * NS], wb[U][2 * NS], sa[U], ba[U], sb[U], bb[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t k_at = at + (16 * u + kg) * S::kRow;
    lds_words<NS>(wa[u], k_at + 8 * NS * t);
    lds_words<NS>(wb[u], k_at + S::kRow + 8 * NS * t);
    const uint32_t pa = lds32(k_at + 32 * NS + 4 * group), pb = lds32(k_at + S::kRow + 32 * NS + 4 * group);
    sa[u] = both_low(pa);
    ba[u] = both_high(pa);
    sb[u] = both_low(pb);
    bb[u] = both_high(pb);
  }
#pragma unroll
  for (int i = 0; i < 2 * NS; ++i) {
    uint32_t q[NT][4];
#pragma unroll
    for (int x = 0; x < NT; ++x) lds_words<2>(q[x], q_at + (x * 2 * NS + i) * 512);
#pragma unroll
    for (int j = 0; j < 4; j += 2)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t a0 = fma16x2<T>(pair4<T>(wa[u][i], j), sa[u], ba[u]), a1 = fma16x2<T>(pair4<T>(wb[u][i], j), sb[u], bb[u]);
        const uint32_t a2 = fma16x2<T>(pair4<T>(wa[u][i], j + 1), sa[u], ba[u]);
        const uint32_t a3 = fma16x2<T>(pair4<T>(wb[u][i], j + 1), sb[u], bb[u]);
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          float(&d)[4] = s[u][x];
          if (i == 0 && j == 0) M::run(d, a0, a1, a2, a3, q[x][j], q[x][j + 1], 0.f, 0.f, 0.f, 0.f);
          else M::run(d, a0, a1, a2, a3, q[x][j], q[x][j + 1], d[0], d[1], d[2], d[3]);
        }
      }
  }
  // weights; s[u][x][0], [1]: key kg of query rows 2 t and 2 t + 1, [2], [3]: the key after
  if ((int32_t)(key0 + 16 * U) > least) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if ((int32_t)(key0 + 16 * u + kg + (k >> 1)) >= see[x][k & 1]) s[u][x][k] = -INFINITY;
  }
  float p[U][NT][4], most = 0.f;
  auto weigh = [&] {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          p[u][x][k] = exp2_approx(fmaf(s[u][x][k], sl2, M::kShift - st.top[x][k & 1]));
          most = fmaxf(most, p[u][x][k]);
        }
  };
  weigh();
  if (__any_sync(kFull, most > kMove4 * M::kScale)) {
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float mx = fmaxf(fmaxf(s[0][x][y], s[0][x][y + 2]), fmaxf(s[U - 1][x][y], s[U - 1][x][y + 2])) * sl2;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, o));
        const float top = st.top[x][y], up = fmaxf(top, mx), f = exp2_approx(top - up);
        st.top[x][y] = up;
        st.l[x][y] *= f;
#pragma unroll
        for (int i = 0; i < 4 * NS; ++i) {
          st.o[x][i][y] *= f;
          st.o[x][i][y + 2] *= f;
        }
      }
    weigh();
  }
  const uint32_t r0 = 2 * t, r1 = ((2 * t + 4) & 7) + 8, v_group = NS == 2 ? g >> 1 : g >> 2;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t b[NT][2];
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      st.l[x][0] += p[u][x][0] + p[u][x][2];
      st.l[x][1] += p[u][x][1] + p[u][x][3];
      b[x][0] = transposed(M::pack(p[u][x][0], p[u][x][1]));
      b[x][1] = transposed(M::pack(p[u][x][2], p[u][x][3]));
    }
    // values: keys 2 t and 2 t + 1 of the matrix's order, and the two 8 rows on
    const uint32_t v0 = at + S::kTensor + (16 * u + r0) * S::kRow, v1 = at + S::kTensor + (16 * u + r1) * S::kRow;
    uint32_t w[4][NS], par[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t row = (k & 1 ? v1 : v0) + (k >> 1) * S::kRow;
      lds_half<NS>(w[k], row + 4 * NS * g);
      par[k] = lds32(row + 32 * NS + 4 * v_group);
    }
    if (key0 + 16 * u + 16 > n) {  // slots that hold no token may hold anything: values of 0
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (key0 + 16 * u + (k & 1 ? r1 : r0) + (k >> 1) >= n) par[k] = 0;
    }
    const uint32_t s0 = __byte_perm(par[0], par[1], 0x5410), b0 = __byte_perm(par[0], par[1], 0x7632);
    const uint32_t s1 = __byte_perm(par[2], par[3], 0x5410), b1 = __byte_perm(par[2], par[3], 0x7632);
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const uint32_t e0 = __byte_perm(w[0][i], w[1][i], 0x5410), d0 = __byte_perm(w[0][i], w[1][i], 0x7632);
      const uint32_t e1 = __byte_perm(w[2][i], w[3][i], 0x5410), d1 = __byte_perm(w[2][i], w[3][i], 0x7632);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t a0 = fma16x2<T>(pair4<T>(e0, j), s0, b0), a1 = fma16x2<T>(pair4<T>(d0, j), s0, b0);
        const uint32_t a2 = fma16x2<T>(pair4<T>(e1, j), s1, b1), a3 = fma16x2<T>(pair4<T>(d1, j), s1, b1);
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          float(&d)[4] = st.o[x][4 * i + j];
          M::run(d, a0, a1, a2, a3, b[x][0], b[x][1], d[0], d[1], d[2], d[3]);
        }
      }
    }
  }
}

// A row's parts put together, `count` of them: part p is at slot(p).  By a warp.
template <typename T, int NS, int NT>
__device__ __noinline__ void join_row(const Few4Args& a, uint32_t c0, uint32_t count, uint32_t row, uint64_t at) {
  using S = Shape<NS, NT>;
  const uint32_t lane = threadIdx.x & 31, D = a.kv.D;
  auto slot = [&](uint32_t p) { return 2 * (uint64_t)(c0 + p) + (p == 0 ? 1 : 0); };
  float top = -INFINITY, l = 0.f;
  for (uint32_t p = lane; p < count; p += 32) top = fmaxf(top, __ldcg(a.part_ml + slot(p) * S::kQRows + row).x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
  float4 o4 = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool in = 4 * lane < S::kDim;
  for (uint32_t p0 = 0; p0 < count; p0 += 32) {
    float f = 0.f;
    if (p0 + lane < count) {
      const float2 ml = __ldcg(a.part_ml + slot(p0 + lane) * S::kQRows + row);
      f = ml.x == -INFINITY ? 0.f : exp2_approx(ml.x - top);
      l += ml.x == -INFINITY ? 0.f : ml.y * f;
    }
    const uint32_t some = count - p0 < 32 ? count - p0 : 32;
#pragma unroll 8
    for (uint32_t p = 0; p < some; ++p) {
      const float4 x = in ? __ldcg(reinterpret_cast<const float4*>(a.part + (slot(p0 + p) * S::kQRows + row) * S::kDim) + lane)
                          : make_float4(0.f, 0.f, 0.f, 0.f);
      const float fp = __shfl_sync(kFull, f, p);
      if (fp == 0.f) continue;  // the row saw no key of the part
      o4.x = fmaf(x.x, fp, o4.x);
      o4.y = fmaf(x.y, fp, o4.y);
      o4.z = fmaf(x.z, fp, o4.z);
      o4.w = fmaf(x.w, fp, o4.w);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(kFull, l, o);
  const bool none = top == -INFINITY;
  const float inv = none ? 0.f : 1.f / l;
  if (4 * lane < D)
    *reinterpret_cast<uint2*>(a.out + 2 * (at * D + 4 * lane)) =
        make_uint2(Mma16<T>::pack(o4.x * inv, o4.y * inv), Mma16<T>::pack(o4.z * inv, o4.w * inv));
  if (lane == 0) a.lse[at] = none ? -INFINITY : (top + log2_approx(l)) * kLn2;
}

template <typename T, int NS, int NT, bool BLOCKS>
__device__ __forceinline__ void take_units(const Few4Args& a, Shared& sh, Way& w, bool more, char* smem, uint64_t all,
                                           uint32_t ctas) {
  using S = Shape<NS, NT>;
  using M = Mma16<T>;
  const uint32_t tid = threadIdx.x, warp = warp_index(), lane = tid & 31, g = lane >> 2, t = lane & 3, team = warp / kTeam;
  const uint32_t D = a.kv.D, G = a.G;
  const float sl2 = a.scale * kLog2e;
  const uint32_t ring = smem_u32(smem) + warp * S::kRing * S::kStage;
  char* rows = smem + S::kRows0;
  uint4* queries = reinterpret_cast<uint4*>(smem + S::kQueries0);
  const uint32_t q_at = smem_u32(queries + lane);
  Feed<NS, NT, BLOCKS> feed;
  feed.begin(a, sh, w, more);
#pragma unroll
  for (uint32_t i = 0; i + 1 < S::kRing; ++i) feed.issue(a, sh, ring);
  uint32_t item = 0;
  for (; more; more = w.next(a, sh)) {
    // the queries' operand, once for all warps: lane (g, t) of it has, of row 8 x + g,
    // channels 16 NS t on, eight a piece
    for (uint32_t x = warp; x < 2 * NS * NT; x += kWarps) {
      const uint32_t i = 8 * (x / (2 * NS)) + g, d = 16 * NS * t + 8 * (x % (2 * NS)), tok = i / G;
      uint4 y = make_uint4(0, 0, 0, 0);
      if (tok < w.m && d < D)
        y = *reinterpret_cast<const uint4*>(a.q + 2 * ((int64_t)(w.tok0 + tok) * a.q_tok + (int64_t)(w.h * G + i % G) * a.q_head + d));
      queries[x * 32 + lane] = y;
    }
    int32_t see[NT][2];
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (uint32_t y = 0; y < 2; ++y) {  // keys that query row 8 x + 2 t + y sees (rows that are none: all)
        const uint32_t mine = (8 * x + 2 * t + y) / G;
        const int64_t last = (int64_t)w.n - w.m + mine + 1;
        see[x][y] = mine >= w.m ? (int32_t)w.n : last > 0 ? (int32_t)last : 0;
      }
    const int32_t least = w.n >= w.m ? (int32_t)(w.n - w.m + 1) : 0;
    __syncthreads();
    Rows<NS, NT> st;
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        st.top[x][y] = kNoTop;
        st.l[x][y] = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * NS; ++i) st.o[x][i][y] = st.o[x][i][y + 2] = 0.f;
      }
    const uint32_t chunks = (w.kv1 - w.kv0) * (kUnit / kChunk);
    for (uint32_t c = warp; c < chunks; c += kWarps, ++item) {
      const uint32_t key0 = w.kv0 * kUnit + c * kChunk;
      cp_async_wait<S::kRing - 2>();
      __syncwarp();  // the chunk is there for all lanes, and all are through with the one before
      feed.issue(a, sh, ring);
      const uint32_t at = ring + item % S::kRing * S::kStage;
#pragma unroll
      for (uint32_t u = 0; u < 2; u += S::kBlocks)
        if (key0 + 16 * u < w.n)
          take_keys<T, NS, NT, S::kBlocks>(at + 16 * u * S::kRow, key0 + 16 * u, w.n, see, least, sl2, q_at, st);
    }
    // the warps' rows: the second team's are added to the first's
    char* region = rows + (warp % kTeam) * S::kRegion;
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) st.l[x][y] += __shfl_xor_sync(kFull, st.l[x][y], o);
    float4* mine = reinterpret_cast<float4*>(region) + lane;
    if (team == 1) {
#pragma unroll
      for (int x = 0; x < NT; ++x) {
#pragma unroll
        for (int i = 0; i < 4 * NS; ++i)
          mine[32 * (x * (4 * NS + 1) + i)] = make_float4(st.o[x][i][0], st.o[x][i][1], st.o[x][i][2], st.o[x][i][3]);
        mine[32 * (x * (4 * NS + 1) + 4 * NS)] = make_float4(st.top[x][0], st.top[x][1], st.l[x][0], st.l[x][1]);
      }
    }
    __syncthreads();
    if (team == 0) {
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const float4 o = mine[32 * (x * (4 * NS + 1) + 4 * NS)];
        const float top[2] = {fmaxf(st.top[x][0], o.x), fmaxf(st.top[x][1], o.y)};
        const float f[2] = {exp2_approx(st.top[x][0] - top[0]), exp2_approx(st.top[x][1] - top[1])};
        const float h[2] = {exp2_approx(o.x - top[0]), exp2_approx(o.y - top[1])};
        st.l[x][0] = st.l[x][0] * f[0] + o.z * h[0];
        st.l[x][1] = st.l[x][1] * f[1] + o.w * h[1];
        st.top[x][0] = top[0];
        st.top[x][1] = top[1];
#pragma unroll
        for (int i = 0; i < 4 * NS; ++i) {
          const float4 y = mine[32 * (x * (4 * NS + 1) + i)];
          st.o[x][i][0] = fmaf(st.o[x][i][0], f[0], y.x * h[0]);
          st.o[x][i][1] = fmaf(st.o[x][i][1], f[1], y.y * h[1]);
          st.o[x][i][2] = fmaf(st.o[x][i][2], f[0], y.z * h[0]);
          st.o[x][i][3] = fmaf(st.o[x][i][3], f[1], y.w * h[1]);
        }
      }
      __syncwarp();  // the region is the warp's own from here on
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t i = 8 * x + 2 * t + y;
          const float l = st.l[x][y];
          if (g == 0) sh.ml[warp][i] = make_float2(l != 0.f ? st.top[x][y] - M::kShift : -INFINITY, l);
          float4* to = reinterpret_cast<float4*>(reinterpret_cast<float*>(region) + i * S::kORow + 8 * NS * g);
#pragma unroll
          for (int k = 0; k < 2 * NS; ++k)
            to[k] = make_float4(st.o[x][2 * k][y], st.o[x][2 * k][y + 2], st.o[x][2 * k + 1][y], st.o[x][2 * k + 1][y + 2]);
        }
    }
    __syncthreads();
    const bool whole = w.kv0 == 0 && w.kv1 == w.tiles;
    const uint32_t used = w.m * G;
    const uint64_t out0 = w.tok0 * a.n_q_heads + w.h * G;  // of row 0; row i is token i / G, head i % G
    const uint64_t slot = 2 * (uint64_t)blockIdx.x + (w.kv0 ? 0 : 1);
    constexpr uint32_t kAcross = S::kDim / 4;
    for (uint32_t e = tid; e < S::kQRows * kAcross; e += 32 * kWarps) {
      const uint32_t i = e / kAcross, c = 4 * (e % kAcross);
      if (i >= used) break;
      float top = -INFINITY, l = 0.f;
#pragma unroll
      for (uint32_t x = 0; x < kTeam; ++x) top = fmaxf(top, sh.ml[x][i].x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (uint32_t x = 0; x < kTeam; ++x) {
        const float2 ml = sh.ml[x][i];
        if (ml.x == -INFINITY) continue;
        const float f = exp2_approx(ml.x - top);
        const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(rows + x * S::kRegion) + i * S::kORow + c);
        l = fmaf(ml.y, f, l);
        o.x = fmaf(y.x, f, o.x);
        o.y = fmaf(y.y, f, o.y);
        o.z = fmaf(y.z, f, o.z);
        o.w = fmaf(y.w, f, o.w);
      }
      if (whole) {
        const bool none = top == -INFINITY;
        const float inv = none ? 0.f : 1.f / l;
        const uint64_t to = out0 + (uint64_t)(i / G) * a.n_q_heads + i % G;
        if (c < D)
          *reinterpret_cast<uint2*>(a.out + 2 * (to * D + c)) =
              make_uint2(M::pack(o.x * inv, o.y * inv), M::pack(o.z * inv, o.w * inv));
        if (c == 0) a.lse[to] = none ? -INFINITY : (top + log2_approx(l)) * kLn2;
      } else {
        *reinterpret_cast<float4*>(a.part + (slot * S::kQRows + i) * S::kDim + c) = o;
        if (c == 0) a.part_ml[slot * S::kQRows + i] = make_float2(top, l);
      }
    }
    if (!whole) {
      // the CTAs that share the tile: those of its first and its last key, and all between
      const uint64_t first = w.tile0 + kExtra;
      const uint32_t c0 = (uint32_t)(((first + 1) * ctas + all - 1) / all - 1);
      const uint32_t c1 = (uint32_t)(((first + w.tiles) * ctas + all - 1) / all - 1);
      __threadfence();
      __syncthreads();
      if (tid == 0) sh.last = atomicAdd(a.arrived + c0, 1u) == c1 - c0;
      __syncthreads();
      if (sh.last) {
        __threadfence();
        for (uint32_t i = warp; i < used; i += kWarps)
          join_row<T, NS, NT>(a, c0, c1 - c0 + 1, i, out0 + (uint64_t)(i / G) * a.n_q_heads + i % G);
      }
    }
    __syncthreads();
  }
  cp_async_wait<0>();
}

template <typename T, int NS, int NT, bool BLOCKS>
__global__ void __launch_bounds__(kThreads, Shape<NS, NT>::kCtas) k_attn4_few(const __grid_constant__ Few4Args a) {
  using S = Shape<NS, NT>;
  extern __shared__ __align__(128) char smem_raw[];
  __shared__ Shared sh;
  grid_dep_sync();
  uint64_t all;
  if (!add_up(a, sh, all)) return;
  const uint32_t ctas = all < a.ctas ? (uint32_t)all : a.ctas;  // every CTA has a unit
  if (blockIdx.x >= ctas) return;
  Way w;
  const bool more = w.begin(a, sh, all, blockIdx.x, ctas);
  take_units<T, NS, NT, BLOCKS>(a, sh, w, more, smem_raw, all, ctas);
}

template <typename T, int NS, int NT, bool BLOCKS>
ptc_status launch_one(const Few4Args& a, cudaStream_t s) {
  constexpr int smem = Shape<NS, NT>::kBytes;
  static std::atomic<uint64_t> ready{0};
  const auto kernel = k_attn4_few<T, NS, NT, BLOCKS>;
  if (!large_smem(kernel, smem, ready)) return PTC_ERR_CUDA;
  PTC_KERNEL("k_attn4_few", s, kernel, a.ctas, kThreads, smem, a);
  return PTC_OK;
}
template <typename T>
ptc_status launch_some(const Few4Args& a, uint32_t rows, bool blocks, cudaStream_t s) {
#define PTC_FEW4(NS, NT) (blocks ? launch_one<T, NS, NT, true>(a, s) : launch_one<T, NS, NT, false>(a, s))
  if (a.kv.D > 64) return rows > 16 ? PTC_FEW4(2, 4) : rows > 8 ? PTC_FEW4(2, 2) : PTC_FEW4(2, 1);
  return rows > 16 ? PTC_FEW4(1, 4) : rows > 8 ? PTC_FEW4(1, 2) : PTC_FEW4(1, 1);
#undef PTC_FEW4
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

uint32_t padded_rows(uint32_t rows) { return rows > 16 ? 32 : rows > 8 ? 16 : 8; }
uint32_t few4_ctas(uint32_t head_dim, uint32_t rows) {
  const uint32_t n = (uint32_t)num_sms() * (padded4(head_dim) / 64 * padded_rows(rows) <= 16 ? 2 : 1);
  return n < kFew4MaxCtas ? n : kFew4MaxCtas;
}

}  // namespace

size_t few4_ws(uint32_t head_dim, uint32_t rows) {
  const size_t places = 2 * (size_t)few4_ctas(head_dim, rows) * padded_rows(rows);
  return up256(4 * kFew4MaxCtas) + up256(8 * places) + up256(4 * places * padded4(head_dim));
}

ptc_status launch_few4(const AttnArgs& c, uint32_t rows, char* ws, bool bf16, cudaStream_t s) {
  Few4Args a{c.kv, c.q, c.q_tok, c.q_head, c.tok_off, c.n_tok, c.n_q_heads, c.G, c.max_q_len, c.scale, c.out, c.lse};
  a.status = c.status;
  a.ctas = few4_ctas(a.kv.D, rows);
  const size_t places = 2 * (size_t)a.ctas * padded_rows(rows);
  a.arrived = reinterpret_cast<uint32_t*>(ws);
  ws += up256(4 * kFew4MaxCtas);
  a.part_ml = reinterpret_cast<float2*>(ws);
  a.part = reinterpret_cast<float*>(ws + up256(8 * places));
  const int64_t row = row4_bytes(a.kv.D);
  // (places in the cache by 16 are numbers of 32 bits then)
  const int64_t most = a.kv.ks_page > a.kv.vs_page ? a.kv.ks_page : a.kv.vs_page;
  const bool blocks = a.kv.B % 16 == 0 && a.kv.ks_slot == row && a.kv.vs_slot == row &&
                      most <= (int64_t(1) << 36) / ((int64_t)a.kv.n_pages + 1);
  a.k_page16 = (uint32_t)(a.kv.ks_page / 16);
  a.v_page16 = (uint32_t)(a.kv.vs_page / 16);
  page_division(a.kv.B, &a.div_mul, &a.div_shift);
  const ptc_status st = fill_async(a.arrived, 0u, 4 * a.ctas, s);
  if (st != PTC_OK) return st;
  return bf16 ? launch_some<__nv_bfloat16>(a, rows, blocks, s) : launch_some<__half>(a, rows, blocks, s);
}

}  // namespace ptc
