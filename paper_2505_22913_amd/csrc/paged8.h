// Internal interface of the paged cache in 8 bits (paged8_api.hip and its kernels in paged8.hip
// and paged8_attn.hip) and of rotary positions (rope.hip).
#pragma once

#include "mustafar.h"
#include "paged.h"

namespace mf {

struct Paged8View {
  PagedView p;  // k and v: codes, a byte each; bf16: the type of tokens, queries and outputs
  uint8_t* k_scale;
  uint8_t* v_scale;
  int int8;  // codes are int8, else e4m3
  int log2_block;
};

hipError_t launch_paged8_write(const Paged8View& c, const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new,
                               int64_t v_stride, const int32_t* cu, int n_new, hipStream_t s);
hipError_t launch_paged8_gather(const Paged8View& c, const int32_t* first, uint16_t* x_k, uint16_t* x_v, int n_max,
                                hipStream_t s);

// p.k and p.v are the codes, p.bf16 the type of q and out.
struct Paged8AttnArgs : PagedAttnArgs {
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  int int8, log2_block;
  // Ranges of a kv-head in a launch of k_paged8_rows that shares `budget` of them out among the requests by their lengths (flat, the
  // launch's, is more where there are more tiles of rows; 0: `few` ranges of every request). info: for each row where its results
  // begin and how many ranges they are of.
  int64_t flat;
  int budget;
  int2* info;
};

// As PagedPlan; `few` is 2 where there are `flat` ranges.
struct Paged8Plan : PagedPlan {
  int64_t flat;
  int budget;
};
// Waves of k_paged8_rows, where requests are divided, and the tokens of a range from which they are shared out by the requests' lengths.
// (A wave looks at all requests then, eight a lane at most.)
constexpr int kFew8Waves = 1024, kFlat8Tokens = 768, kFlat8Requests = 512;

// Rows of the ranges' results of k_paged8_rows, 16 of each of `flat`.
template <class Plan>
inline int64_t paged8_few_rows(const PagedView& p, const Plan& k, int64_t few_rows) {
  return k.flat ? k.flat * p.H * kFewRows : paged_parts(few_rows, k.few);
}
inline int64_t paged8_parts(const Paged8AttnArgs& a, int64_t few_rows) { return paged8_few_rows(a.p, a, few_rows); }

struct Kernels8 {
  using Plan = Paged8Plan;
  static Plan choose(const PagedView& p, int G, int n_q, int max_q, int64_t max_tokens, int n_splits) {
    Plan k;
    static_cast<PagedPlan&>(k) = paged_kernels(p, G, n_q, max_q, max_tokens, n_splits);
    k.flat = 0;
    k.budget = 0;
    if (k.few == 0 || n_splits > 0) return k;
    // Tiles of rows of a kv-head (as paged_kernels counts them, and how many there can be).
    const int64_t requests = p.B < n_q ? p.B : n_q, full = k.mixed ? 0 : ((int64_t)n_q * G + kFewRows - 1) / kFewRows;
    const int64_t units = requests > full ? requests : full, most_units = requests + (k.mixed ? 0 : (int64_t)n_q * G / kFewRows);
    const int64_t n = kFew8Waves / (units * p.H), most = max_tokens / 64;
    k.few = (int)(n < 1 || most < 1 ? 1 : n < most ? n : most);
    // (Over kFew8Waves / 2 tiles of rows and kv-heads a wave each, whatever the requests' lengths, which the host does not know: 24 requests of
    // 8192 tokens with 32 heads take 251 us, 6.4 TB/s, and 263 where two waves a SIMD are shared out; of lengths from an eighth up to that
    // 239 and 176. 96 requests with 8 heads 251 and 264, 240 and 186.)
    if (k.few == 1 || requests == 1 || max_tokens < kFlat8Tokens * k.few || p.B > kFlat8Requests) return k;
    k.few = 2;
    k.budget = kFew8Waves / p.H;
    k.flat = k.budget > most_units ? k.budget : most_units;
    return k;
  }
  static int64_t ws_bytes(const PagedView& p, int64_t rows, const Plan& k) {
    return (paged8_few_rows(p, k, k.few_rows) + paged_parts(rows, k.most_many)) * (p.d + 2) * 4 + (k.flat ? 8 * k.few_rows : 0);
  }
  static double few_groups(const PagedView& p, const Plan& k, int64_t tiles) {
    return k.flat ? (double)k.flat * p.H : (double)tiles * p.H * k.few;
  }
};
hipError_t launch_paged8_attn(const Paged8AttnArgs& a, hipStream_t s);

// Blocks of tokens that hold the n_new rows of B requests, however they are divided, and k_paged8_write's workgroups for one: a wave
// has 16 tokens of a head's keys or values, the waves of a block lie in one workgroup.
constexpr int kWrite8Threads = 256, kWrite8Rows = 16;
inline int64_t paged8_blocks(const PagedView& p, int log2_block, int n_new) {
  return ((int64_t)n_new >> log2_block) + 2 * (int64_t)p.B;
}
inline int paged8_block_groups(const PagedView& p, int log2_block) {
  const int heads = kWrite8Threads / kWaveSize * kWrite8Rows >> log2_block;  // of keys and values, a workgroup
  return (2 * p.H + heads - 1) / heads;
}

struct RopeArgs {
  const double* rates;
  int rot, layout;
  float magnitude;
  int bf16, inverse;
  const uint16_t* q;
  const uint16_t* k;
  uint16_t* out_q;
  uint16_t* out_k;
  int64_t q_stride, k_stride, out_q_stride, out_k_stride;
  int Hq, H, d, n;
  const int32_t* positions;  // or cu and state
  const int32_t* cu;
  const int32_t* state;
  int B;
  int64_t most;  // tokens that an entry can hold
};
// A workgroup of k_rope: kRopeTokens tokens of so many heads, each row in `pieces` of 16 bytes, the `turned` ones first (in place: those
// alone).
constexpr int kRopeThreads = 256, kRopeTokens = 4, kRopeHeads = 8, kMaxRopeHeads = 1 << 16;
struct RopePlan {
  int width;  // 8: a piece and the one rot / 2 channels on are turned together; 0: pieces hold their pairs; 4, 2 or 1: so many channels
              // and those rot / 2 on, in LDS
  int heads, head_groups;
  int turned, pieces, units;  // units: of `width` pairs, of a row
  // x / head_groups = x * groups_inverse >> 40 (x < 2^24, head_groups <= 2^14); x / pieces = x * pieces_inverse >> 24, and so for units
  // (x < 2^14, pieces and units under 2^8).
  uint64_t groups_inverse;
  uint32_t pieces_inverse, units_inverse;
  int64_t groups;
};
inline RopePlan rope_plan(const RopeArgs& a) {
  const int all = a.Hq + a.H, pairs = a.rot / 2, whole = (a.rot + 7) & ~7;
  RopePlan r;
  const bool in_place = (a.Hq == 0 || a.out_q == a.q) && (a.H == 0 || a.out_k == a.k);
  r.width = a.layout != MUSTAFAR_ROPE_HALF ? 0 : pairs % 8 == 0 ? 8 : pairs % 4 == 0 ? 4 : pairs % 2 == 0 ? 2 : 1;
  r.turned = r.width == 8 ? pairs / 8 : whole / 8;
  r.pieces = r.turned + (in_place ? 0 : (a.d - whole) / 8);
  r.units = r.width ? pairs / r.width : 1;
  // (9600 tokens of 40 heads of 128: 42.0 us with 4 heads, 38.3 with 8, 37.7 with 16, where 64 tokens take 3.6 us for 3.1; 20 of 80
  // channels of 4096 tokens of 64 heads: 21.1 with 5, 19.8 with 8, 19.1 with 12, 25 with 16)
  r.heads = all < kRopeHeads ? all : kRopeHeads;
  r.head_groups = (all + r.heads - 1) / r.heads;
  r.groups = ((int64_t)a.n + kRopeTokens - 1) / kRopeTokens * r.head_groups;
  r.groups_inverse = ((uint64_t)1 << 40) / (uint64_t)r.head_groups + 1;
  r.pieces_inverse = (1u << 24) / (uint32_t)r.pieces + 1;
  r.units_inverse = (1u << 24) / (uint32_t)r.units + 1;
  return r;
}

hipError_t launch_rope(const RopeArgs& a, const RopePlan& plan, hipStream_t s);

}  // namespace mf
