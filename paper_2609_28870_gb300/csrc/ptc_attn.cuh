// Attention over pages: what its kernels share (ptc_attn.cu: plan, tiles,
// join, the C entry point; ptc_mass.cu: the accumulated weights).
#pragma once

#include "ptc_kv.cuh"
#include "ptc_tc.cuh"

namespace ptc {

// The G query heads of a key head are packed as rows of one matrix, token by
// token, so that a key tile is read once for all of them.  128 rows hold
// tq = 128 / G whole tokens; a query tile is two such halves.
constexpr uint32_t kRows = 256, kKeys = 128;
constexpr uint32_t kMassKeys = 256;  // keys of a tile of the weights' kernel
constexpr uint32_t kMaxGroup = PTC_MAX_GROUP;
constexpr uint32_t kMaxCtas = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Where a CTA starts: its first unit, and what that is: for the tile kernel
// the key tile `minor` of query tile `major`, for the weights the query tile
// `minor` (after the first one that sees it) of key tile `major`.
struct CtaStart {
  uint64_t u, tok0, page0;  // tok0, page0, m, n: of request r
  uint32_t r, h, major, minor, m, n;
};

// What k_attn_plan leaves for the kernels after it.  Their work is a row of
// units: for every request, key head and first-level tile (a query tile, or a
// key tile for the weights) `extra` units for what a tile costs by itself, then
// one for every pair with a second-level tile.  CTA c of C takes the units from
// start[c].u to start[c + 1].u, about U / C of them: a cut that falls among the
// extra units or would leave a short part is moved to before or after the tile
// (there, `minor` is past its last second-level tile).
struct AttnPlan {
  uint32_t ok, pad;
  CtaStart start[kMaxCtas + 1];
  uint32_t arrived[kMaxCtas];  // parts of the split tile that begins in CTA c
};

struct AttnArgs {
  KvView kv;
  const char* q;
  int64_t q_tok, q_head;
  const uint64_t* tok_off;
  uint64_t n_tok;
  uint32_t n_q_heads, G, max_q_len;
  uint32_t tq, tq32;   // whole tokens in 128 and in 32 rows
  float scale;
  char* out;
  float* lse;
  const float* mass_in;
  float* mass_out;
  uint64_t mass_stride;
  AttnPlan* plan;      // [0] tiles, [1] weights
  uint64_t* unit_off;  // twice n_req + 1
  float* part;         // unnormalised rows of split tiles: [2 * ctas][kRows][D]
  float2* part_ml;     // their maxima (in powers of two) and sums
  float* part_mass;    // weights of split key tiles: [2 * ctas][kMassKeys]
  float* scores;       // scores of few rows, [n_kv_heads][few][slots], or null
  uint32_t few;
  uint32_t ctas, box;  // box: rows of a tensor copy of keys or values
  uint32_t most;       // tokens of a request
  uint32_t div_mul, div_shift;  // key / B for pages of 4 bits; see page_division
  uint32_t withhold;   // test of the bounded waits: no queries are loaded
  long long limit;     // cycles after which a wait for another role gives up
  uint32_t* status;
};

// Units that a tile costs by itself (the softmax's first steps, the sums' way
// out).  A step of mixed chunks took 549, 494, 489 and 500 us with 1, 2, 3 and 5
// for every tile, 64 single tokens 179, 182, 185 and 191 us: a tile of few rows
// costs one key tile, any other three.  (A key tile counts the same under a short
// query tile: counted as half of one, the mixed chunks took 524 us, not 468.)  A
// key tile's sum of weights costs about one query tile.
constexpr uint32_t kTileExtra = 3, kFewExtra = 1, kMassExtra = 1;
// Fewest key tiles of a part.  A part of up to 256 rows costs their sums' way
// through memory (6 us for two parts of 256 rows); one of few rows hardly any.
constexpr uint32_t kPartMin = 4;

// The CTAs that share the units [from, to) of a split tile, c0 the first.
struct Sharers {
  uint32_t c0, c1, count;
};
// By a whole warp, over the plan's starts.
__device__ __forceinline__ Sharers sharers(const AttnPlan* plan, uint32_t ctas, uint64_t from, uint64_t to) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t before = 0, until = 0, inside = 0;
  for (uint32_t x = lane; x < ctas; x += 32) {
    const uint64_t u = plan->start[x].u, v = plan->start[x + 1].u;
    before += u <= from;
    until += u < to;
    inside += u > from && u < to && v > u;
  }
  before = __reduce_add_sync(kFull, before);
  until = __reduce_add_sync(kFull, until);
  inside = __reduce_add_sync(kFull, inside);
  return {before - 1, until - 1, inside + 1};
}

__host__ __device__ __forceinline__ uint32_t div_up(uint32_t a, uint32_t b) { return (a + b - 1) / b; }

// Query tiles of `span` tokens of a request, and the key tiles that one of them
// sees, at least one.
__device__ __forceinline__ uint32_t key_tiles(uint32_t m, uint32_t n, uint32_t span, uint32_t qt) {
  const uint32_t end = (qt + 1) * span < m ? (qt + 1) * span : m;
  const int64_t sees = (int64_t)n - m + end;
  return sees <= (int64_t)kKeys ? 1u : (uint32_t)((sees + kKeys - 1) / kKeys);
}
// What query tile qt costs by itself.
__device__ __forceinline__ uint32_t tile_extra(uint32_t m, uint32_t span, uint32_t tq32, uint32_t qt) {
  return m - qt * span <= tq32 ? kFewExtra : kTileExtra;
}
// The first half tile of queries that sees anything of the weights' key tile kt.
__device__ __forceinline__ uint32_t first_seeing(uint32_t m, uint32_t n, uint32_t tq, uint32_t kt) {
  const int64_t t = (int64_t)kt * kMassKeys - ((int64_t)n - m);
  return t <= 0 ? 0u : (uint32_t)t / tq;
}

// Host side (ptc_attn.cu, ptc_mass.cu).
// Workspace: the status word, the plans, the unit offsets, the parts, the scores.
struct AttnWs {
  size_t plan, units, ml, part, mass, scores, total;
};
AttnWs attn_ws(uint32_t n_req, uint32_t ctas, uint32_t D, uint64_t scores);
uint32_t tile_ctas();
void attn_place(AttnArgs& a, const AttnWs& at, char* ws);
// What a call says of its queries: checks, and what follows from them.
ptc_status attn_call(AttnArgs& a, const ptc_paged_kv* kv, const uint64_t* tok_off, uint64_t n_tok, const int64_t* q_stride,
                     uint32_t n_q_heads, float scale);
ptc_status attn_rows(AttnArgs& a, const void* q, const int64_t* q_stride, uint32_t max_q_len, void* out, float* lse);
void launch_plan(const AttnArgs& a, bool weights, cudaStream_t s);
// The whole call over pages of 16 bits, after its checks.
ptc_status launch_attention(AttnArgs& a, bool bf16, cudaStream_t s);
bool tokens_map(CUtensorMap* map, const AttnArgs& a, bool bf16, uint32_t tokens);
bool cache_map(CUtensorMap* map, const KvView& kv, bool bf16, char* base, int64_t page, int64_t head, int64_t slot,
               uint32_t box);
// Most rows of a request whose scores are kept for the weights; see ptc_mass.cu.
constexpr uint32_t kFewRows = 16;
ptc_status launch_mass(const AttnArgs& a, bool bf16, const CUtensorMap& mk, const CUtensorMap& mq, bool tma,
                       cudaStream_t s);

}  // namespace ptc
