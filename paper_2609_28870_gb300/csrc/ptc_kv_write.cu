// New tokens on their way into the pages, turned and quantised
// (ptc_kv_append_rope, ptc_kv4_append), and back (ptc_kv4_read).
#include <type_traits>

#include "ptc_kv4.cuh"

namespace ptc {
namespace {

constexpr int kWrThreads = 256;
constexpr int kRdRows = 4;  // rows of a token that a thread has in flight, of those that are read back
constexpr uint32_t kWrSlice = 48;

struct WriteArgs {
  KvView kv;
  RopeView rope;
  const char* q;
  char* q_out;
  int64_t q_tok, q_head, o_tok, o_head;
  const char* kn;
  const char* vn;
  int64_t kn_tok, kn_head, vn_tok, vn_head;
  char* k_out;  // of ptc_kv4_read
  char* v_out;
  const uint64_t* tok_off;
  uint64_t n_tok;
  uint32_t n_q_heads, slice, rows;  // rows of a token, and those that a CTA takes
  uint32_t* status;
};

// Where a token's row of head 0 lies in the pages, or k = -1, and its position.
struct Place {
  int64_t k, v;
  uint32_t pos;
};

// The first CTA of a call looks whether the offsets are in order.
__device__ __forceinline__ void check_offsets(const WriteArgs& a) {
  if (blockIdx.x || blockIdx.y) return;
  bool bad = threadIdx.x == 0 && (a.tok_off[0] != 0 || a.tok_off[a.kv.n_req] != a.n_tok);
  for (uint32_t r = threadIdx.x; r < a.kv.n_req; r += kWrThreads) bad |= a.tok_off[r] > a.tok_off[r + 1];
  if (bad) report(a.status, PTC_ERR_INVALID_ARG);
}

__device__ __forceinline__ Place find_place(const WriteArgs& a, uint64_t t) {
  Place at{-1, -1, 0};
  const uint32_t r = req_search(a.tok_off, 0, a.kv.n_req - 1, t);
  const uint64_t lo = a.tok_off[r], hi = a.tok_off[r + 1];
  const uint64_t n = a.kv.kv_len[r];
  if (lo <= t && t < hi && hi <= a.n_tok && hi - lo <= n && pages_hold(a.kv, r, n)) {
    const uint64_t j = n - (hi - t);
    const uint32_t page = a.kv.page_ids[a.kv.page_off[r] + j / a.kv.B];
    const int64_t slot = (int64_t)(j % a.kv.B);
    at.pos = a.rope.pos ? a.rope.pos[t] : (uint32_t)j;
    if (page < a.kv.n_pages && (!a.rope.table || at.pos < a.rope.n_pos)) {
      at.k = (int64_t)page * a.kv.ks_page + slot * a.kv.ks_slot;
      at.v = (int64_t)page * a.kv.vs_page + slot * a.kv.vs_slot;
    }
  }
  if (at.k < 0) report(a.status, PTC_ERR_INVALID_ARG);
  return at;
}

template <uint32_t TOKENS>
__device__ __forceinline__ void find_places(const WriteArgs& a, uint64_t t0, Place (&at)[TOKENS]) {
  check_offsets(a);
  if (threadIdx.x < TOKENS) at[threadIdx.x] = t0 + threadIdx.x < a.n_tok ? find_place(a, t0 + threadIdx.x) : Place{-1, -1, 0};
  __syncthreads();
}

// How a call turns its rows: not at all; neighbours, or channels of the two halves,
// in whole threads (the pairs a multiple of 4, of 8); any other number of pairs
// (neighbours whose pairs are no multiple of 4, halves whose pairs are none of 8).  A
// kernel each: one for all of them, whose registers the rarest width decides, took 140
// us for 138 below, in fp16 160 for 140, into 4 bits 203 for 194 (fp16 226 for 203).
enum Width { kStill, kNext, kHalves, kAnyWidth };

// CTAs of an SM.  With four a thread has 64 registers, which do not hold all it needs: up
// to 44 bytes of it are stored and loaded again, of kAnyWidth up to 68, in fp16 164.
// There three are faster (50 pairs in halves 226 -> 214 us, in neighbours 173 -> 164, 36 in
// halves 175 -> 165; in bf16 197 -> 201, 147 -> 156, 149 -> 158).
template <typename T>
constexpr int write_ctas(Width width) {
  return width == kAnyWidth && !Half16<T>::kBf16 ? 3 : 4;
}

// How a thread's eight channels are turned: by the same angles for all heads of
// a token, so they are kept.  sn has its sign: channel e becomes
// x[e] cs[e] + partner sn[e].
struct Turn {
  float2 cs[4], sn[4];
  uint32_t mask[4];  // the channels that are turned, where not all are
  bool any, all;
};

template <Width WIDTH>
__device__ __forceinline__ void load_turn(const RopeView& rope, uint32_t pos, uint32_t c, Turn& o) {
  const uint32_t F = rope.n_freq, d0 = 8 * c;
  const float* row = rope.table + (uint64_t)pos * 2 * F;
  o.any = d0 < 2 * F;
  o.all = F % 4 == 0;  // 2 F is a multiple of 8
  if (!o.any) return;
  if (WIDTH == kNext) {
    const float4 x = __ldg(reinterpret_cast<const float4*>(row + 4 * c)), y = __ldg(reinterpret_cast<const float4*>(row + F + 4 * c));
    const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      o.cs[k] = make_float2(xs[k], xs[k]);
      o.sn[k] = make_float2(-ys[k], ys[k]);
    }
  } else if (WIDTH == kHalves || F % 4 == 0) {
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
      const uint32_t d = d0 + 4 * k, i = d < F ? d : d - F;
      const float sign = d < F ? -1.f : 1.f;
      const float4 x = __ldg(reinterpret_cast<const float4*>(row + i)), y = __ldg(reinterpret_cast<const float4*>(row + F + i));
      o.cs[2 * k] = make_float2(x.x, x.y);
      o.cs[2 * k + 1] = make_float2(x.z, x.w);
      o.sn[2 * k] = make_float2(sign * y.x, sign * y.y);
      o.sn[2 * k + 1] = make_float2(sign * y.z, sign * y.w);
    }
  } else {
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      float cs[2] = {1.f, 1.f}, sn[2] = {0.f, 0.f};
      o.mask[k] = 0;
#pragma unroll
      for (uint32_t e = 0; e < 2; ++e) {
        const uint32_t d = d0 + 2 * k + e;
        if (d >= 2 * F) continue;
        const uint32_t i = rope.interleaved ? d / 2 : d < F ? d : d - F;
        const bool second = rope.interleaved ? d & 1 : d >= F;
        o.mask[k] |= 0xFFFFu << (16 * e);
        cs[e] = __ldg(row + i);
        const float s = __ldg(row + F + i);
        sn[e] = second ? s : -s;
      }
      o.cs[k] = make_float2(cs[0], cs[1]);
      o.sn[k] = make_float2(sn[0], sn[1]);
    }
  }
}

// The partners of channels d0 on, one by one; those of channels that are not turned
// are themselves.
__device__ __forceinline__ uint4 partners_apart(const char* row, uint32_t d0, uint32_t F, uint4 x) {
  uint32_t p[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t d = d0 + e;
    if (d < 2 * F) {
      const uint32_t y = *reinterpret_cast<const uint16_t*>(row + 2 * (d < F ? d + F : d - F));
      p[e / 2] = e & 1 ? (p[e / 2] & 0xFFFFu) | y << 16 : (p[e / 2] & 0xFFFF0000u) | y;
    }
  }
  return make_uint4(p[0], p[1], p[2], p[3]);
}

// A row's channels turned; x: the thread's eight, row: all of them in global
// memory.  By all lanes of the row (c: the lane's place among them).
template <typename T, int LANES, Width WIDTH>
__device__ __forceinline__ uint4 turn_row(const RopeView& rope, const Turn& t, const uint4& x, const char* row, uint32_t c,
                                          bool live) {
  const uint32_t F = rope.n_freq;
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t p[4] = {x.x, x.y, x.z, x.w};
  if (WIDTH == kNext || (WIDTH == kAnyWidth && rope.interleaved)) {
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = __byte_perm(w[k], w[k], 0x1032);
  } else if (WIDTH == kHalves) {
    const uint32_t f = F / 8, other = c < f ? c + f : c < 2 * f ? c - f : c;
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = __shfl_sync(kFull, w[k], other, LANES);
  } else if (F % 4 == 0) {  // half a thread's channels on: its lower four have another's upper ones for partners
    auto other = [&](uint32_t d) { return (d < F ? d + F : d < 2 * F ? d - F : d) / 8; };
    const uint32_t l0 = other(8 * c), l1 = other(8 * c + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = __shfl_sync(kFull, w[k ^ 2], k < 2 ? l0 : l1, LANES);
  } else if (live && t.any) {
    const uint4 y = partners_apart(row, 8 * c, F, x);
    p[0] = y.x;
    p[1] = y.y;
    p[2] = y.z;
    p[3] = y.w;
  }
  if (!t.any) return x;
  uint32_t o[4] = {w[0], w[1], w[2], w[3]};
  turn8<T>(o, p, t.cs, t.sn);
  if (WIDTH == kAnyWidth && !t.all) {
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = (o[k] & t.mask[k]) | (w[k] & ~t.mask[k]);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// What 32 bits do not settle of a group's scale, its base and a code.  (Inlined,
// these were computed for every group and picked from afterwards, at the 64-bit
// unit's sixtieth of the rate.)
template <typename T>
__device__ __noinline__ T scale_wide(float lo, float hi) {
  return Half16<T>::put(((double)hi - (double)lo) / 15.0);
}
template <typename T>
__device__ __noinline__ T base_wide(float lo, float s) {
  return Half16<T>::put((double)lo - 16.0 * (double)s);
}
// Whether 32-bit numbers divided by s stay clear of the ends of their range: 31 s,
// the most that a value is above its base, is not infinite, nor 1 / s cut off.
__device__ __forceinline__ bool plain_scale(float s) {
  return __float_as_uint(s) - __float_as_uint(0x1p-100f) <= __float_as_uint(0x1p100f) - __float_as_uint(0x1p-100f);
}
// Eight codes, where 32 bits do not hold what is taken from b.
template <typename T>
__device__ __noinline__ uint32_t codes_wide(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, float b, float s) {
  const uint32_t w[4] = {w0, w1, w2, w3};
  const float inv = 1.f / s, half = 0.5f * s;
  uint32_t code = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 pair = Half16<T>::get2(w[e / 2]);
    const float v = e & 1 ? pair.y : pair.x, y = v - b, z = y - v;
    const float lost = (v - (y - z)) + (-b - z);  // of y by its rounding
    float k = fminf(fmaxf(rintf(fmaf(y, inv, -16.f)), 0.f), 15.f);
    const float r = fmaf(-(k + 16.f), s, y);
    k += (r > half || (r == half && lost >= 0.f) ? 1.f : 0.f) - (r < -half || (r == -half && lost < 0.f) ? 1.f : 0.f);
    if (!plain_scale(s)) k = (float)floor(((double)v - (double)b) / (double)s - 15.5);
    code |= (uint32_t)fminf(fmaxf(k, 0.f), 15.f) << (4 * (e / 2) + 16 * (e & 1));
  }
  return code;
}

// The codes of eight channels, and their group's scale and base.  A group is
// four threads' channels; a thread without channels (real = false) takes part.
template <typename T>
__device__ __forceinline__ uint32_t quantise(const uint4& x, bool real, uint32_t& words) {
  using Two = typename Half16<T>::Two;
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  auto two = [](uint32_t v) { return *reinterpret_cast<const Two*>(&v); };
  auto raw = [](Two v) { return *reinterpret_cast<const uint32_t*>(&v); };
  constexpr uint32_t kInf2 = Half16<T>::kBf16 ? 0x7F807F80u : 0x7C007C00u;
  // the smallest and the largest with its sign changed, in one word; NaN stays
  const Two small = __hmin2_nan(__hmin2_nan(two(w[0]), two(w[1])), __hmin2_nan(two(w[2]), two(w[3])));
  const Two large = __hmax2_nan(__hmax2_nan(two(w[0]), two(w[1])), __hmax2_nan(two(w[2]), two(w[3])));
  const uint32_t a = raw(small), b = raw(large) ^ 0x80008000u;
  uint32_t m = raw(__hmin2_nan(two(__byte_perm(a, b, 0x5410)), two(__byte_perm(a, b, 0x7632))));
  if (!real) m = kInf2;
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) m = raw(__hmin2_nan(two(m), two(__shfl_xor_sync(kFull, m, o))));
  const float2 ends = Half16<T>::get2(m);
  const float lo = ends.x, hi = -ends.y;
  words = 0;
  if (m == kInf2) return 0;  // no channel in the group (an infinity among them makes the other end finite or -infinity)
  // (three roundings of half a unit: within 3 units in the last place)
  const float d = hi - lo, s32 = d * (1.f / 15.f);
  const T s = Half16<T>::unsure(s32) || !(d < INFINITY) ? scale_wide<T>(lo, hi) : Half16<T>::put(s32);
  const float sf = Half16<T>::get(s), s16 = 16.f * sf;
  const bool near = lo == 0.f || (fabsf(lo) >= Half16<T>::kExact * s16 && s16 >= Half16<T>::kExact * fabsf(lo));
  const T base = near && s16 < INFINITY ? Half16<T>::put(lo - s16) : base_wide<T>(lo, sf);
  const float bf = Half16<T>::get(base);
  if (!(sf < INFINITY) || !(fabsf(bf) < INFINITY)) {
    words = Half16<T>::kBf16 ? 0x7FC07FC0u : 0x7E007E00u;
    return 0;
  }
  words = bits16(s) | bits16(base) << 16;
  if (sf == 0.f || !real) return 0;
  // y / s, of y = v - b, to the nearest whole number in a sum's last bits, with a
  // reciprocal a few units too large: so what lies on a code's border goes up, as it
  // should.  y less that many s, exact, tells of a value that lies so close below a border
  // that it went up too (more than half an s away), and of one on it: there what y's
  // subtraction lost in 32 bits matters, where value and base are far apart in size.
  uint32_t code = 0;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(sf));
  inv = fmaf(inv, 0x1p-21f, inv);
  constexpr float kSum = 12582912.f - 16.f;  // 1.5 * 2^23: whole numbers; the base absorbs 16
  const float half = 0.5f * sf;
  const float most = fmaxf(fmaxf(fabsf(lo), fabsf(hi)), fabsf(bf)), least = Half16<T>::kExact * most;
  const bool fine = plain_scale(sf) && (bf == 0.f || fabsf(bf) >= least);
  float away = 0.f, small_v = INFINITY;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = Half16<T>::get2(w[i]), y = add2(v, both(-bf));
    const float2 z = fma2(y, both(inv), both(kSum)), k = add2(z, both(-kSum)), r = fma2(k, both(-sf), y);
    away = fmaxf(away, fmaxf(fabsf(r.x), fabsf(r.y)));
    small_v = fminf(small_v, fminf(fabsf(v.x), fabsf(v.y)));
    code |= __vimin_s16x2_relu(__byte_perm(__float_as_uint(z.x), __float_as_uint(z.y), 0x5410), 0x000F000F) << (4 * i);
  }
  if (!fine || away > half || (away == half && small_v < least)) code = codes_wide<T>(w[0], w[1], w[2], w[3], bf, sf);
  return code;
}

// The rows of tokens: queries, keys and values, LANES threads a row with eight
// channels each (so that a row stays within a warp: it may be turned in place).
// A group of LANES threads stays with its token and takes `slice` of its rows, so that
// the token's place and angles are found once for them; queries, keys and values in a
// loop each, with what it needs in registers and no more (a loop over rows of all
// kinds: 152 us for 140, into 4 bits 223 for 203).  Each row is read and written once,
// 0.86 GB for 34,692 tokens of 32 query and 8 key heads of 128: 138 us, 6.2 TB/s; into
// pages of 4 bits 158 us, bound by its instructions.  (Several batches of tokens a CTA,
// to wait for places less often, were slower by 6%.)  Halves of no multiple of 8
// pairs 148 us, of no multiple of 4 197 us.  64 tokens 4.3 us, a launch and four
// dependent reads.
template <typename T, int LANES, bool FOUR, Width WIDTH>
__global__ void __launch_bounds__(kWrThreads, write_ctas<T>(WIDTH)) k_kv_write(const __grid_constant__ WriteArgs a) {
  grid_dep_sync();
  constexpr uint32_t kTok = kWrThreads / LANES;
  __shared__ Place s_at[kTok];
  const uint64_t t0 = (uint64_t)blockIdx.x * kTok;
  find_places(a, t0, s_at);
  const Place at = s_at[threadIdx.x / LANES];
  const int64_t t = (int64_t)t0 + threadIdx.x / LANES;
  const uint32_t c = threadIdx.x % LANES, D = a.kv.D, Hq = a.n_q_heads, H = a.kv.H;
  const bool live = at.k >= 0, real = 8 * c < D;
  constexpr bool turned = WIDTH != kStill;
  Turn angles;
  angles.any = false;
  if (turned && live && real) load_turn<WIDTH>(a.rope, at.pos, c, angles);
  const uint32_t first = blockIdx.y * a.slice, end = first + a.slice < a.rows ? first + a.slice : a.rows;
  // n rows, a stride apart where they come from and where they go to; ROWS of them are
  // worked on while as many are loaded.
  auto take = [&](auto rows_at_once, auto quantised, bool turn, const char* from, int64_t from_step, char* to, int64_t step,
                  uint32_t n) {
    constexpr uint32_t ROWS = decltype(rows_at_once)::value;
    constexpr bool QUANT = decltype(quantised)::value;
    uint4 x[ROWS], next[ROWS];
    auto load = [&](uint32_t r, uint32_t ahead) {
      return r < n && live && real ? *reinterpret_cast<const uint4*>(from + ahead * from_step + 16 * c) : make_uint4(0, 0, 0, 0);
    };
#pragma unroll
    for (uint32_t u = 0; u < ROWS; ++u) next[u] = load(u, u);
#pragma unroll 1
    for (uint32_t r0 = 0; r0 < n; r0 += ROWS) {
#pragma unroll
      for (uint32_t u = 0; u < ROWS; ++u) {
        x[u] = next[u];
        next[u] = load(r0 + ROWS + u, ROWS + u);
      }
#pragma unroll
      for (uint32_t u = 0; u < ROWS; ++u) {
        if (r0 + u >= n) break;  // the whole CTA
        uint4 y = x[u];
        if (turn) y = turn_row<T, LANES, WIDTH>(a.rope, angles, x[u], from, c, live);
        __syncwarp();  // a row is written after all of it was read
        if (!QUANT) {
          if (live && real) *reinterpret_cast<uint4*>(to + 16 * c) = y;
        } else {
          uint32_t words;
          const uint32_t code = quantise<T>(y, live && real, words);
          if (live) {
            uint32_t* row = reinterpret_cast<uint32_t*>(to);
            row[c] = code;
            if (c % 4 == 0) row[LANES + c / 4] = words;
            if (LANES == 8 && c % 4 == 1) row[10 + c / 4] = 0;
          }
        }
        from += from_step;
        to += step;
      }
    }
  };
  // The CTA's rows of a kind, of which `before` rows are of others.
  constexpr int64_t kUnit = FOUR ? 1 : 2;  // bytes of a stride's unit in the pages
  using Now = std::integral_constant<uint32_t, FOUR ? 1 : 2>;
  auto part = [&](uint32_t before, uint32_t rows, uint32_t& r) {
    const uint32_t lo = first > before ? first - before : 0, hi = end > before ? end - before : 0;
    r = lo < rows ? lo : rows;
    return (hi < rows ? hi : rows) - r;
  };
  uint32_t r, n;
  if ((n = part(0, Hq, r)) > 0)
    take(std::integral_constant<uint32_t, 2>{}, std::false_type{}, turned, a.q + 2 * (t * a.q_tok + r * a.q_head), 2 * a.q_head,
         a.q_out + 2 * (t * a.o_tok + r * a.o_head), 2 * a.o_head, n);
  if ((n = part(Hq, H, r)) > 0)
    take(Now{}, std::integral_constant<bool, FOUR>{}, turned, a.kn + 2 * (t * a.kn_tok + r * a.kn_head), 2 * a.kn_head,
         a.kv.k + kUnit * (at.k + r * a.kv.ks_head), kUnit * a.kv.ks_head, n);
  if ((n = part(Hq + H, H, r)) > 0)
    take(std::integral_constant<uint32_t, FOUR ? 2 : 4>{}, std::integral_constant<bool, FOUR>{}, false,
         a.vn + 2 * (t * a.vn_tok + r * a.vn_head), 2 * a.vn_head, a.kv.v + kUnit * (at.v + r * a.kv.vs_head), kUnit * a.kv.vs_head, n);
}

// Tokens back out of their pages: 0.46 GB in 73 us, 6.3 TB/s, at HBM's rate.
template <typename T, int LANES>
__global__ void __launch_bounds__(kWrThreads) k_kv4_read(const __grid_constant__ WriteArgs a) {
  grid_dep_sync();
  constexpr uint32_t kTok = kWrThreads / LANES;
  __shared__ Place s_at[kTok];
  const uint64_t t0 = (uint64_t)blockIdx.x * kTok;
  find_places(a, t0, s_at);
  const Place at = s_at[threadIdx.x / LANES];
  const uint64_t t = t0 + threadIdx.x / LANES;
  const uint32_t c = threadIdx.x % LANES, D = a.kv.D, H = a.kv.H;
  if (at.k < 0 || 8 * c >= D) return;
  const uint32_t first = blockIdx.y * a.slice, end = first + a.slice < a.rows ? first + a.slice : a.rows;
  for (uint32_t r0 = first; r0 < end; r0 += kRdRows) {
    uint32_t w[kRdRows], p[kRdRows];
#pragma unroll
    for (int u = 0; u < kRdRows; ++u) {
      const uint32_t r = r0 + u < end ? r0 + u : end - 1;
      const bool key = r < H;
      const char* row = key ? a.kv.k + at.k + r * a.kv.ks_head : a.kv.v + at.v + (r - H) * a.kv.vs_head;
      w[u] = *reinterpret_cast<const uint32_t*>(row + 4 * c);
      p[u] = *reinterpret_cast<const uint32_t*>(row + 4 * (LANES + c / 4));
    }
#pragma unroll
    for (int u = 0; u < kRdRows; ++u) {
      const uint32_t r = r0 + u;
      if (r >= end) break;
      const uint32_t s = both_low(p[u]), b = both_high(p[u]);
      const uint4 y = make_uint4(fma16x2<T>(pair4<T>(w[u], 0), s, b), fma16x2<T>(pair4<T>(w[u], 1), s, b),
                                 fma16x2<T>(pair4<T>(w[u], 2), s, b), fma16x2<T>(pair4<T>(w[u], 3), s, b));
      char* to = r < H ? a.k_out : a.v_out;
      *reinterpret_cast<uint4*>(to + 2 * ((t * H + (r < H ? r : r - H)) * D + 8 * c)) = y;
    }
  }
}

// Rows of a CTA: as few as leave four CTAs for every SM, so that a call of few
// tokens is spread, and at most kWrSlice.  34,692 tokens, turned, and into 4 bits and
// back, us:
//   rows of a CTA, at most           3        6       12       24       48
//   48 rows a token            205 287  163 225  146 199  142 191  138 185
//   12                          57  82   47  66   42  60   42  60   42  60
//   3                           19  31   19  31   19  31   19  31   19  31  (1: 28 45)
dim3 write_grid(WriteArgs& a, uint32_t tok) {
  const uint64_t blocks = (a.n_tok + tok - 1) / tok;
  uint64_t slice = blocks * a.rows / (4 * (uint64_t)num_sms());
  a.slice = (uint32_t)(slice < 1 ? 1 : slice > kWrSlice ? kWrSlice : slice);
  if ((a.rows + a.slice - 1) / a.slice > 65535) a.slice = (a.rows + 65534) / 65535;
  return dim3((uint32_t)blocks, (a.rows + a.slice - 1) / a.slice);
}

template <typename T, bool FOUR, Width WIDTH>
void launch_width(WriteArgs& a, cudaStream_t s) {
  const char* name = FOUR ? "k_kv4_append" : "k_kv_append_rope";
  if (a.kv.D <= 64) PTC_KERNEL(name, s, (k_kv_write<T, 8, FOUR, WIDTH>), write_grid(a, kWrThreads / 8), kWrThreads, 0, a);
  else PTC_KERNEL(name, s, (k_kv_write<T, 16, FOUR, WIDTH>), write_grid(a, kWrThreads / 16), kWrThreads, 0, a);
}
template <typename T, bool FOUR>
void launch_write(WriteArgs& a, cudaStream_t s) {
  const uint32_t F = a.rope.n_freq;
  if (FOUR && !a.rope.table) launch_width<T, FOUR, FOUR ? kStill : kAnyWidth>(a, s);
  else if (a.rope.interleaved && F % 4 == 0) launch_width<T, FOUR, kNext>(a, s);
  else if (!a.rope.interleaved && F % 8 == 0) launch_width<T, FOUR, kHalves>(a, s);
  else launch_width<T, FOUR, kAnyWidth>(a, s);
}
template <typename T>
void launch_read(WriteArgs& a, cudaStream_t s) {
  if (a.kv.D <= 64) PTC_KERNEL("k_kv4_read", s, (k_kv4_read<T, 8>), write_grid(a, kWrThreads / 8), kWrThreads, 0, a);
  else PTC_KERNEL("k_kv4_read", s, (k_kv4_read<T, 16>), write_grid(a, kWrThreads / 16), kWrThreads, 0, a);
}

// What ptc_kv_append_rope and ptc_kv4_append have in common.
template <bool FOUR>
ptc_status write_tokens(const ptc_paged_kv* kv, const ptc_rope* rope, const void* q, const int64_t q_stride[2], void* q_out,
                        const int64_t q_out_stride[2], uint32_t n_q_heads, const void* k_new, const void* v_new,
                        const int64_t k_new_stride[2], const int64_t v_new_stride[2], const uint64_t* tok_off, uint64_t n_tok,
                        void* ws, size_t ws_bytes, uint32_t* status, void* stream) {
  WriteArgs a{};
  ptc_status st = FOUR ? kv4_view(kv, &a.kv) : kv_view(kv, &a.kv);
  if (st == PTC_OK && rope) st = rope_view(rope, kv->head_dim, &a.rope);
  if (st != PTC_OK) return st;
  if (!tok_off || !k_new_stride || !v_new_stride || (n_tok && !kv->n_req) || (n_q_heads && (!rope || !q_stride || !q_out_stride)))
    return PTC_ERR_INVALID_ARG;
  if (n_q_heads > 65535u * PTC_MAX_GROUP) return PTC_ERR_INVALID_ARG;
  if (n_tok > (uint64_t(1) << 31)) return PTC_ERR_OVERFLOW;
  if (!status && !ws_ok(ws, ws_bytes, kKvStatusBytes)) return PTC_ERR_WORKSPACE;
  if (n_tok == 0) return PTC_OK;
  if (!aligned16(k_new) || !aligned16(v_new) || (n_q_heads && (!aligned16(q) || !aligned16(q_out)))) return PTC_ERR_INVALID_ARG;
  const uint32_t ext[2] = {(uint32_t)n_tok, kv->n_kv_heads}, q_ext[2] = {(uint32_t)n_tok, n_q_heads};
  for (int i = 0; i < 2; ++i) {
    if (!stride_ok(k_new_stride[i], ext[i]) || !stride_ok(v_new_stride[i], ext[i])) return PTC_ERR_INVALID_ARG;
    if (n_q_heads && (!stride_ok(q_stride[i], q_ext[i]) || !stride_ok(q_out_stride[i], q_ext[i]))) return PTC_ERR_INVALID_ARG;
    if (n_q_heads && q == q_out && q_ext[i] > 1 && q_stride[i] != q_out_stride[i]) return PTC_ERR_INVALID_ARG;
  }
  if (rope && !rope->n_pos) return PTC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  a.n_q_heads = n_q_heads;
  if (n_q_heads) {
    a.q = static_cast<const char*>(q);
    a.q_out = static_cast<char*>(q_out);
    a.q_tok = stride_of(q_stride[0], q_ext[0]);
    a.q_head = stride_of(q_stride[1], q_ext[1]);
    a.o_tok = stride_of(q_out_stride[0], q_ext[0]);
    a.o_head = stride_of(q_out_stride[1], q_ext[1]);
  }
  a.kn = static_cast<const char*>(k_new);
  a.vn = static_cast<const char*>(v_new);
  a.kn_tok = stride_of(k_new_stride[0], ext[0]);
  a.kn_head = stride_of(k_new_stride[1], ext[1]);
  a.vn_tok = stride_of(v_new_stride[0], ext[0]);
  a.vn_head = stride_of(v_new_stride[1], ext[1]);
  a.tok_off = tok_off;
  a.n_tok = n_tok;
  a.rows = n_q_heads + 2 * kv->n_kv_heads;
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  if (kv->dtype == PTC_DTYPE_BF16) launch_write<__nv_bfloat16, FOUR>(a, s);
  else launch_write<__half, FOUR>(a, s);
  return kv_end(status, a.status, s);
}

}  // namespace
}  // namespace ptc

using namespace ptc;

extern "C" uint32_t ptc_kv4_row_bytes(uint32_t head_dim) { return row4_bytes(head_dim); }
extern "C" size_t ptc_kv_append_rope_workspace_bytes(uint32_t) { return kKvStatusBytes; }
extern "C" size_t ptc_kv4_append_workspace_bytes(uint32_t) { return kKvStatusBytes; }
extern "C" size_t ptc_kv4_read_workspace_bytes(uint32_t) { return kKvStatusBytes; }

extern "C" ptc_status ptc_kv_append_rope(const ptc_paged_kv* kv, const ptc_rope* rope, const void* q,
                                         const int64_t q_stride[2], void* q_out, const int64_t q_out_stride[2],
                                         uint32_t n_q_heads, const void* k_new, const void* v_new,
                                         const int64_t k_new_stride[2], const int64_t v_new_stride[2],
                                         const uint64_t* tok_off, uint64_t n_tok, void* ws, size_t ws_bytes,
                                         uint32_t* status, void* stream) {
  if (!rope) return PTC_ERR_INVALID_ARG;
  return write_tokens<false>(kv, rope, q, q_stride, q_out, q_out_stride, n_q_heads, k_new, v_new, k_new_stride, v_new_stride,
                             tok_off, n_tok, ws, ws_bytes, status, stream);
}

extern "C" ptc_status ptc_kv4_append(const ptc_paged_kv* kv, const ptc_rope* rope, const void* q, const int64_t q_stride[2],
                                     void* q_out, const int64_t q_out_stride[2], uint32_t n_q_heads, const void* k_new,
                                     const void* v_new, const int64_t k_new_stride[2], const int64_t v_new_stride[2],
                                     const uint64_t* tok_off, uint64_t n_tok, void* ws, size_t ws_bytes,
                                     uint32_t* status, void* stream) {
  return write_tokens<true>(kv, rope, q, q_stride, q_out, q_out_stride, n_q_heads, k_new, v_new, k_new_stride, v_new_stride,
                            tok_off, n_tok, ws, ws_bytes, status, stream);
}

extern "C" ptc_status ptc_kv4_read(const ptc_paged_kv* kv, const uint64_t* tok_off, uint64_t n_tok, void* k_out, void* v_out,
                                   void* ws, size_t ws_bytes, uint32_t* status, void* stream) {
  WriteArgs a{};
  const ptc_status st = kv4_view(kv, &a.kv);
  if (st != PTC_OK) return st;
  if (!tok_off || (n_tok && !kv->n_req)) return PTC_ERR_INVALID_ARG;
  if (n_tok > (uint64_t(1) << 31)) return PTC_ERR_OVERFLOW;
  if (!status && !ws_ok(ws, ws_bytes, kKvStatusBytes)) return PTC_ERR_WORKSPACE;
  if (n_tok == 0) return PTC_OK;
  if (!aligned16(k_out) || !aligned16(v_out)) return PTC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  a.k_out = static_cast<char*>(k_out);
  a.v_out = static_cast<char*>(v_out);
  a.tok_off = tok_off;
  a.n_tok = n_tok;
  a.rows = 2 * kv->n_kv_heads;
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  if (kv->dtype == PTC_DTYPE_BF16) launch_read<__nv_bfloat16>(a, s);
  else launch_read<__half>(a, s);
  return kv_end(status, a.status, s);
}
