// Internal interface of the paged dense cache (paged_api.hip and its kernels in
// paged.hip and paged_attn.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mf {

constexpr int64_t kLastLevel = 256 << 20;  // bytes of the last cache

struct PagedView {
  uint16_t* k;
  uint16_t* v;
  int32_t* table;
  int32_t* state;
  int32_t* free_pages;
  int B, H, d, log2_page, n_pages, max_pages;
  int bf16;  // type of k and v
  int64_t page_stride;
  int head_stride, token_stride;  // a page is under 2^31 bytes
};

hipError_t launch_paged_plan(const PagedView& p, const int32_t* keep, const int32_t* new_len, int32_t* state_out,
                             int32_t* cu, int32_t* slots, int n_slots, int32_t* status, hipStream_t s);
hipError_t launch_paged_write(const PagedView& p, const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new,
                              int64_t v_stride, const int32_t* slots, int n_new, hipStream_t s);
hipError_t launch_paged_gather(const PagedView& p, const int32_t* first, uint16_t* x_k, uint16_t* x_v, int n_max,
                               hipStream_t s);

struct PagedAttnArgs {
  PagedView p;
  const uint16_t* q;
  uint16_t* out;
  const int32_t* cu;
  int64_t q_stride, out_stride;
  int n_q, Hq, G;
  int window, sinks;
  float scale_log2;  // score scale times log2(e)
  // Ranges of a request's visible tokens in k_paged_rows and in k_paged_chunk, 0 where that kernel is not run; mixed: the first
  // has the requests of at most kFewRows rows, the second the others, else the one that runs has all.
  int few, many, mixed;
  // Rows of a range's results in k_paged_rows: of q and all its heads, or, by_entry, kFewRows of every entry and kv-head.
  int64_t few_rows;
  int by_entry;
  void* ws;  // the ranges' results where there are several
};

// Rows are a request's new tokens times the query heads of a kv-head. k_paged_rows takes 16 at a time, k_paged_chunk 32 a wave and
// 8 waves a workgroup (4 at d = 256; d = 64 T).
constexpr int kFewRows = 16, kWaveSize = 64;
constexpr int chunk_waves(int T) { return T == 4 ? 4 : 8; }
constexpr int chunk_rows(int T) { return 32 * chunk_waves(T); }
// Workgroups of k_paged_merge with a stream of 16 T lanes a row.
constexpr int kMergeThreads = 256;
inline int64_t merge_groups(int64_t rows, int T) { return (rows * 16 * T + kMergeThreads - 1) / kMergeThreads; }
// Workgroups of so many rows that hold n_q tokens of B requests however they are divided.
inline int64_t paged_tiles(const PagedView& p, int G, int n_q, int rows) { return (int64_t)n_q * G / rows + p.B; }

// Which kernels a call takes, and the ranges that it takes by itself (n_splits <= 0) for requests of up to max_q tokens that see
// up to max_tokens.
struct PagedPlan {
  int few, many, mixed;
  int most_many;  // at least the ranges `many` of this and of every smaller max_tokens (`few` are that themselves)
  int64_t few_rows;
  int by_entry;
};

// Results of the ranges of both kernels: two numbers and d fp32 values of every row. By themselves calls take at most 16 * 2048 and
// 256 * 256 such rows (ranges times rows; the launch's waves and workgroups times theirs), whatever the batch.
inline int64_t paged_parts(int64_t rows, int ranges) { return ranges > 1 ? rows * ranges : 0; }
inline int64_t paged_ws_bytes(const PagedView& p, int64_t rows, const PagedPlan& k) {
  return (paged_parts(k.few_rows, k.few) + paged_parts(rows, k.most_many)) * (p.d + 2) * 4;
}

inline PagedPlan paged_kernels(const PagedView& p, int G, int n_q, int max_q, int64_t max_tokens, int n_splits) {
  PagedPlan k = {0, 0, 0, 0, 0, 0};
  const bool all_few = (int64_t)max_q * G <= kFewRows;
  const bool uneven = p.B > 1 && n_q < (int64_t)p.B * max_q;  // (else every request has max_q)
  k.mixed = !all_few && uneven && G <= kFewRows;
  const int64_t q_rows = (int64_t)n_q * G * p.H, entry_rows = (int64_t)p.B * p.H * kFewRows;
  k.by_entry = k.mixed && entry_rows < q_rows;
  k.few_rows = k.by_entry ? entry_rows : q_rows;
  auto ranges = [&](int64_t groups, int64_t target, int64_t least) {
    if (n_splits > 0) return n_splits;
    const int64_t n = target / groups, most = max_tokens / least;
    return (int)(n < 1 || most < 1 ? 1 : n < most ? n : most);
  };
  // Few rows: waves of at least 64 tokens, one a SIMD (1024). With two a SIMD the long requests of a ragged batch are shared out
  // better, but a range's output costs as much as 2 tokens a row: 16 requests of 16384 tokens on average take 115 us for 125 with
  // lengths from nothing to twice that and 4 rows, 167 for 164 with equal lengths; of 16 rows 185 for 168. Rows of d = 256 cost
  // twice as much (4 of 4 requests of 4096 tokens: 40 for 34).
  const int64_t rows = (all_few ? max_q : 1) * (int64_t)G;
  auto tiles = [&](int64_t tokens, int rows) { return (tokens * G + rows - 1) / rows; };
  if (all_few || k.mixed) {
    const int64_t requests = p.B < n_q ? p.B : n_q, full = all_few ? tiles(n_q, kFewRows) : 0;  // (more than the requests if max_q is too small)
    k.few = ranges((requests > full ? requests : full) * p.H, rows <= 4 && p.d < 256 ? 2048 : 1024, 64);
  }
  // Many: a workgroup a CU of at least 256 tokens, where the tokens that a workgroup is spared are worth what k_paged_merge costs:
  // the launch as much as 200 tokens of a tile of rows, every range of one on a CU as much as 600. 599 tokens and 80 workgroups
  // take 22 us and 32 in two ranges, 1024 and 128 32 and 39; 1536 and 64 41 and 37 in four, 2304 and 128 62 and 59 in two.
  if (!all_few) {
    const int rows = chunk_rows(p.d / 64);
    const int64_t full = tiles(n_q, rows), even = uneven || p.B == 1 ? 0 : p.B * tiles(max_q, rows);
    const int64_t groups = (even > full ? even : full) * p.H;
    k.many = k.most_many = ranges(groups, 256, 256);
    if (n_splits <= 0 && max_tokens - max_tokens / k.many < 200 + 600 * groups * k.many / 256) k.many = 1;
  }
  return k;
}
hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s);

}  // namespace mf
