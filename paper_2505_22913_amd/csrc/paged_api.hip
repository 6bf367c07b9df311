// C ABI of the paged dense cache (declared in include/mustafar.h): host-side checks,
// then the launches. Every check runs before any launch.
#include "paged_host.h"

using namespace mf;

extern "C" {

int mustafar_paged_init(mustafar_pages_t* p, void* k, void* v, void* table, void* state, void* free_pages, int B, int H,
                        int d, int page_tokens, int n_pages, int max_pages, int type, int64_t page_stride,
                        int64_t head_stride, int64_t token_stride) {
  if (!p) return MUSTAFAR_EINVAL;
  mustafar_pages_t t;
  t.k = k;
  t.v = v;
  t.table = (int32_t*)table;
  t.state = (int32_t*)state;
  t.free_pages = (int32_t*)free_pages;
  t.B = B;
  t.H = H;
  t.d = d;
  t.page_tokens = page_tokens;
  t.n_pages = n_pages;
  t.max_pages = max_pages;
  t.type = type;
  t.page_stride = page_stride;
  t.head_stride = head_stride;
  t.token_stride = token_stride;
  const int st = check_pages(&t);
  if (st != MUSTAFAR_OK) return st;
  *p = t;
  return MUSTAFAR_OK;
}

int mustafar_paged_plan(const mustafar_pages_t* p, const void* keep, const void* new_len, void* state_out, void* cu,
                        void* slots, int n_slots, void* status, void* stream) {
  int st = check_any_pages(p);
  if (st != MUSTAFAR_OK) return st;
  if (n_slots < 0 || n_slots > MUSTAFAR_PAGED_MAX_STEP) return MUSTAFAR_EINVAL;
  if (!aligned(new_len, 4) || !aligned(state_out, 4) || !aligned(cu, 4) || !aligned(status, 4)) return MUSTAFAR_EINVAL;
  if ((keep && !aligned(keep, 4)) || (n_slots > 0 && !aligned(slots, 4))) return MUSTAFAR_EINVAL;
  if (state_out != p->state && overlap(state_out, p->state, 4 * ((size_t)p->B + 2))) return MUSTAFAR_EINVAL;
  return status_of(launch_paged_plan(view_of(p), (const int32_t*)keep, (const int32_t*)new_len,
                                         (int32_t*)state_out, (int32_t*)cu, (int32_t*)slots, n_slots,
                                         (int32_t*)status, (hipStream_t)stream));
}

int mustafar_paged_write(const mustafar_pages_t* p, const void* k_new, int64_t k_stride, const void* v_new,
                         int64_t v_stride, const void* slots, int n_new, void* stream) {
  int st = check_pages(p);
  if (st != MUSTAFAR_OK) return st;
  if (n_new < 0) return MUSTAFAR_EINVAL;
  if (n_new == 0) return MUSTAFAR_OK;
  const int64_t row = (int64_t)p->H * p->d;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(slots, 4)) return MUSTAFAR_EINVAL;
  if (k_stride < row || v_stride < row || k_stride % 8 != 0 || v_stride % 8 != 0 || k_stride > (int64_t)1 << 31 ||
      v_stride > (int64_t)1 << 31)
    return MUSTAFAR_EINVAL;
  return status_of(launch_paged_write(view_of(p), (const uint16_t*)k_new, k_stride, (const uint16_t*)v_new,
                                          v_stride, (const int32_t*)slots, n_new, (hipStream_t)stream));
}

int mustafar_paged_gather(const mustafar_pages_t* p, const void* first, void* x_k, void* x_v, int n_max, void* stream) {
  int st = check_pages(p);
  if (st != MUSTAFAR_OK) return st;
  if (n_max < 0) return MUSTAFAR_EINVAL;
  if (n_max == 0) return MUSTAFAR_OK;
  if (!aligned(x_k, 16) || !aligned(x_v, 16) || (first && !aligned(first, 4))) return MUSTAFAR_EINVAL;
  const int64_t groups = ((int64_t)n_max * (p->d / 8) + 255) / 256;  // of an entry and kv-head
  if (!launches((double)p->B * p->H * (double)groups, 256)) return MUSTAFAR_EINVAL;
  return status_of(launch_paged_gather(view_of(p), (const int32_t*)first, (uint16_t*)x_k, (uint16_t*)x_v, n_max,
                                           (hipStream_t)stream));
}

size_t mustafar_paged_attn_workspace_bytes(const mustafar_pages_t* p, int Hq, int n_q, int max_q, int max_tokens,
                                           int n_splits) {
  return check_pages(p) != MUSTAFAR_OK ? 0 : attn_ws_bytes<Kernels16>(view_of(p), Hq, n_q, max_q, max_tokens, n_splits);
}

int mustafar_paged_attn(const void* q, int64_t q_stride, int n_q, int Hq, const mustafar_pages_t* p, const void* cu,
                        int window, int sinks, float scale, void* out, int64_t out_stride, int max_q, int max_tokens,
                        int n_splits, void* ws, size_t ws_bytes, void* stream) {
  int st = check_pages(p);
  if (st != MUSTAFAR_OK) return st;
  PagedAttnArgs a;
  PagedPlan plan;
  st = attn_args<Kernels16>(&a, q, q_stride, n_q, Hq, view_of(p), cu, window, sinks, scale, out, out_stride, max_q, max_tokens,
                            n_splits, ws, ws_bytes, &plan);
  if (st != MUSTAFAR_OK || n_q == 0) return st;
  return status_of(launch_paged_attn(a, (hipStream_t)stream));
}

}  // extern "C"
