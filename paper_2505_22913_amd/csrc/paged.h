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
};
hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s);

}  // namespace mf
