// Internal interface of the paged dense cache (paged_api.hip and its kernels in
// paged.hip and paged_attn.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mf {

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
  int n_splits;      // ranges of a request's visible tokens
  void* ws;          // their results when there are several
};

// Waves of a workgroup, of 32 rows (new tokens times query heads of a kv-head) each; d = 64 T.
constexpr int chunk_waves(int T) { return T == 4 ? 4 : 8; }
// Workgroups that hold the rows of n_q tokens of B requests however they are divided.
inline int64_t paged_tiles(const PagedView& p, int G, int n_q) { return (int64_t)n_q * G / (32 * chunk_waves(p.d / 64)) + p.B; }

// Bytes of the ranges' results: (reference, sum) and d fp32 values of every row and query head.
inline int64_t paged_ws_bytes(const PagedView& p, int Hq, int n_q, int n_splits) {
  return n_splits <= 1 ? 0 : (int64_t)n_splits * n_q * Hq * (p.d + 2) * 4;
}

// Ranges that a call takes by itself: a workgroup a CU, each of at least four tiles.
inline int paged_splits(const PagedView& p, int G, int n_q, int max_q, int64_t max_tokens) {
  const int64_t groups = paged_tiles(p, G, n_q) * p.H, tiles = max_tokens / 64 / 4;
  const int64_t n = 256 / groups;
  return (int)(n < 1 || tiles < 1 ? 1 : n < tiles ? n : tiles);
}
hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s);

}  // namespace mf
