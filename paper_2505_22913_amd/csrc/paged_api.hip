// C ABI of the paged dense cache (declared in include/mustafar.h): host-side checks,
// then the launches. Every check runs before any launch.
#include <math.h>
#include <stdint.h>

#include "mustafar.h"
#include "paged.h"

namespace {

constexpr int kTile = MUSTAFAR_TILE;
constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kMaxSplits = 1 << 16;

bool aligned(const void* p, uintptr_t a) { return p && ((uintptr_t)p % a) == 0; }

// A launch has less than 2^32 threads.
bool launches(double groups, int threads) { return groups * threads < 4294967296.0; }

int status_of(hipError_t e) { return e == hipSuccess ? MUSTAFAR_OK : MUSTAFAR_ELAUNCH; }

int log2_of(int x) {
  int n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

int check_pages(const mustafar_pages_t* p) {
  if (!p || !aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->table, 4) || !aligned(p->state, 4) ||
      !aligned(p->free_pages, 4))
    return MUSTAFAR_EINVAL;
  if (p->B < 1 || p->B > MUSTAFAR_PAGED_MAX_BATCH || p->H < 1) return MUSTAFAR_EINVAL;
  if (p->d != kTile && p->d != 2 * kTile && p->d != 4 * kTile) return MUSTAFAR_EINVAL;
  if (p->page_tokens < 16 || p->page_tokens > 1024 || (p->page_tokens & (p->page_tokens - 1)) != 0)
    return MUSTAFAR_EINVAL;
  if (p->n_pages < 1 || (int64_t)p->n_pages * p->page_tokens > 0x7fffffff) return MUSTAFAR_EINVAL;
  if (p->max_pages < 1 || p->max_pages > MUSTAFAR_PAGED_MAX_STEP) return MUSTAFAR_EINVAL;
  if ((int64_t)p->max_pages * p->page_tokens > 0x7fffffff) return MUSTAFAR_EINVAL;
  if (p->type != MUSTAFAR_FP16 && p->type != MUSTAFAR_BF16) return MUSTAFAR_EINVAL;
  const int64_t most = (int64_t)1 << 30;  // elements of a page: 2^31 bytes
  if (p->head_stride < p->d || p->token_stride < p->d || p->head_stride > most || p->token_stride > most ||
      p->page_stride < p->d || p->page_stride > (int64_t)1 << 40)
    return MUSTAFAR_EINVAL;
  if (p->head_stride % 8 != 0 || p->token_stride % 8 != 0 || p->page_stride % 8 != 0) return MUSTAFAR_EINVAL;
  // the rows of a head, or of a token, and what lies from the first row to the end of the last
  const int64_t of_head = (p->page_tokens - 1) * p->token_stride + p->d, of_token = (p->H - 1) * p->head_stride + p->d;
  if (p->head_stride < of_head && p->token_stride < of_token && p->H > 1) return MUSTAFAR_EINVAL;
  const int64_t extent = of_head + of_token - p->d;
  if (extent >= most || (p->n_pages > 1 && p->page_stride < extent)) return MUSTAFAR_EINVAL;
  return MUSTAFAR_OK;
}

mf::PagedView view_of(const mustafar_pages_t* p) {
  mf::PagedView v;
  v.k = (uint16_t*)p->k;
  v.v = (uint16_t*)p->v;
  v.table = p->table;
  v.state = p->state;
  v.free_pages = p->free_pages;
  v.B = p->B;
  v.H = p->H;
  v.d = p->d;
  v.log2_page = log2_of(p->page_tokens);
  v.n_pages = p->n_pages;
  v.max_pages = p->max_pages;
  v.bf16 = p->type == MUSTAFAR_BF16;
  v.page_stride = p->page_stride;
  v.head_stride = (int)p->head_stride;
  v.token_stride = (int)p->token_stride;
  return v;
}

bool overlap(const void* a, const void* b, size_t bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y ? y - x < bytes : x - y < bytes;
}

}  // namespace

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
  int st = check_pages(p);
  if (st != MUSTAFAR_OK) return st;
  if (n_slots < 0 || n_slots > MUSTAFAR_PAGED_MAX_STEP) return MUSTAFAR_EINVAL;
  if (!aligned(new_len, 4) || !aligned(state_out, 4) || !aligned(cu, 4) || !aligned(status, 4)) return MUSTAFAR_EINVAL;
  if ((keep && !aligned(keep, 4)) || (n_slots > 0 && !aligned(slots, 4))) return MUSTAFAR_EINVAL;
  if (state_out != p->state && overlap(state_out, p->state, 4 * ((size_t)p->B + 2))) return MUSTAFAR_EINVAL;
  return status_of(mf::launch_paged_plan(view_of(p), (const int32_t*)keep, (const int32_t*)new_len,
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
  return status_of(mf::launch_paged_write(view_of(p), (const uint16_t*)k_new, k_stride, (const uint16_t*)v_new,
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
  return status_of(mf::launch_paged_gather(view_of(p), (const int32_t*)first, (uint16_t*)x_k, (uint16_t*)x_v, n_max,
                                           (hipStream_t)stream));
}

size_t mustafar_paged_attn_workspace_bytes(const mustafar_pages_t* p, int Hq, int n_q, int max_q, int max_tokens,
                                           int n_splits) {
  if (check_pages(p) != MUSTAFAR_OK || Hq < 1 || Hq % p->H != 0 || Hq / p->H > MUSTAFAR_PAGED_MAX_GROUP) return 0;
  if (n_q < 1 || max_q < 0 || max_tokens < 0 || n_splits > kMaxSplits || (int64_t)n_q * Hq >= kMaxRows) return 0;
  const mf::PagedView v = view_of(p);
  const mf::PagedPlan k = mf::paged_kernels(v, Hq / p->H, n_q, max_q, max_tokens, n_splits);
  return (size_t)mf::paged_ws_bytes(v, (int64_t)n_q * Hq, k);
}

int mustafar_paged_attn(const void* q, int64_t q_stride, int n_q, int Hq, const mustafar_pages_t* p, const void* cu,
                        int window, int sinks, float scale, void* out, int64_t out_stride, int max_q, int max_tokens,
                        int n_splits, void* ws, size_t ws_bytes, void* stream) {
  int st = check_pages(p);
  if (st != MUSTAFAR_OK) return st;
  if (Hq < 1 || Hq % p->H != 0 || n_q < 0 || max_q < 0 || max_tokens < 0 || window < 0 || sinks < 0)
    return MUSTAFAR_EINVAL;
  if (Hq / p->H > MUSTAFAR_PAGED_MAX_GROUP) return MUSTAFAR_EUNSUPPORTED;
  if (n_q == 0) return MUSTAFAR_OK;
  const int64_t row = (int64_t)Hq * p->d;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(cu, 4)) return MUSTAFAR_EINVAL;
  if (q_stride < row || out_stride < row || q_stride % 8 != 0 || out_stride % 8 != 0 || q_stride > (int64_t)1 << 31 ||
      out_stride > (int64_t)1 << 31)
    return MUSTAFAR_EINVAL;
  if ((int64_t)n_q * Hq >= kMaxRows) return MUSTAFAR_EINVAL;
  if (n_splits > kMaxSplits) return MUSTAFAR_EINVAL;
  mf::PagedAttnArgs a;
  a.p = view_of(p);
  const size_t need = mustafar_paged_attn_workspace_bytes(p, Hq, n_q, max_q, max_tokens, n_splits);
  if (need > 0 && (!aligned(ws, 16) || ws_bytes < need)) return MUSTAFAR_EWORKSPACE;
  // (what the rows see: never more than the workspace was sized for)
  const int64_t seen = window > 0 ? (int64_t)window + max_q + sinks : max_tokens;
  const mf::PagedPlan k = mf::paged_kernels(a.p, Hq / p->H, n_q, max_q, seen < max_tokens ? seen : max_tokens, n_splits);
  const int T = p->d / kTile;
  const int64_t q_rows = (int64_t)n_q * Hq, few_rows = k.mixed ? (int64_t)p->B * p->H * mf::kFewRows : q_rows;
  const int64_t few = k.mixed ? p->B : mf::paged_tiles(a.p, Hq / p->H, n_q, mf::kFewRows);
  const int64_t many = mf::paged_tiles(a.p, Hq / p->H, n_q, mf::chunk_rows(T));
  if (!launches((double)few * p->H * k.few, mf::kWaveSize) || !launches((double)many * p->H * k.many, mf::kWaveSize * mf::chunk_waves(T)))
    return MUSTAFAR_EINVAL;
  if ((k.few > 1 && !launches((double)mf::merge_groups(few_rows, T), mf::kMergeThreads)) ||
      (k.many > 1 && !launches((double)mf::merge_groups(q_rows, T), mf::kMergeThreads)))
    return MUSTAFAR_EINVAL;
  a.few = k.few;
  a.many = k.many;
  a.mixed = k.mixed;
  a.few_rows = k.few_rows;
  a.by_entry = k.by_entry;
  a.ws = ws;
  a.q = (const uint16_t*)q;
  a.out = (uint16_t*)out;
  a.cu = (const int32_t*)cu;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.n_q = n_q;
  a.Hq = Hq;
  a.G = Hq / p->H;
  a.window = window;
  a.sinks = sinks;
  const double s = scale > 0.f ? (double)scale : 1.0 / sqrt((double)p->d);
  a.scale_log2 = (float)(s * 1.4426950408889634);
  return status_of(mf::launch_paged_attn(a, (hipStream_t)stream));
}

}  // extern "C"
