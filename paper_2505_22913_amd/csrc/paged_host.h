// Host-side checks that the C ABIs over pages share (paged_api.hip, paged8_api.hip).
#pragma once

#include <math.h>
#include <stdint.h>

#include "mustafar.h"
#include "paged.h"

namespace mf {

constexpr int kTileChannels = MUSTAFAR_TILE;
constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kMaxSplits = 1 << 16;

inline bool aligned(const void* p, uintptr_t a) { return p && ((uintptr_t)p % a) == 0; }

// A launch has less than 2^32 threads.
inline bool launches(double groups, int threads) { return groups * threads < 4294967296.0; }

inline int status_of(hipError_t e) { return e == hipSuccess ? MUSTAFAR_OK : MUSTAFAR_ELAUNCH; }

inline int log2_of(int x) {
  int n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

// Pages of 16-bit values, or of codes (the descriptor inside one of 8-bit pages, which only a plan takes by itself).
inline bool is_16bit(int type) { return type == MUSTAFAR_FP16 || type == MUSTAFAR_BF16; }
inline bool is_code(int type) { return type == MUSTAFAR_E4M3 || type == MUSTAFAR_INT8; }

inline int check_any_pages(const mustafar_pages_t* p) {
  if (!p || !aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->table, 4) || !aligned(p->state, 4) ||
      !aligned(p->free_pages, 4))
    return MUSTAFAR_EINVAL;
  if (p->B < 1 || p->B > MUSTAFAR_PAGED_MAX_BATCH || p->H < 1) return MUSTAFAR_EINVAL;
  if (p->d != kTileChannels && p->d != 2 * kTileChannels && p->d != 4 * kTileChannels) return MUSTAFAR_EINVAL;
  if (p->page_tokens < 16 || p->page_tokens > 1024 || (p->page_tokens & (p->page_tokens - 1)) != 0)
    return MUSTAFAR_EINVAL;
  if (p->n_pages < 1 || (int64_t)p->n_pages * p->page_tokens > 0x7fffffff) return MUSTAFAR_EINVAL;
  if (p->max_pages < 1 || p->max_pages > MUSTAFAR_PAGED_MAX_STEP) return MUSTAFAR_EINVAL;
  if ((int64_t)p->max_pages * p->page_tokens > 0x7fffffff) return MUSTAFAR_EINVAL;
  if (!is_16bit(p->type) && !is_code(p->type)) return MUSTAFAR_EINVAL;
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

inline int check_pages(const mustafar_pages_t* p) {
  const int st = check_any_pages(p);
  return st == MUSTAFAR_OK && !is_16bit(p->type) ? MUSTAFAR_EINVAL : st;
}

inline PagedView view_of(const mustafar_pages_t* p) {
  PagedView v;
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

inline bool overlap(const void* a, const void* b, size_t bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y ? y - x < bytes : x - y < bytes;
}

// ------------------------------------------------------------------------------------------
// Attention: the arguments of both kinds of pages; `kernels` chooses theirs.
// ------------------------------------------------------------------------------------------
struct Kernels16 {
  using Plan = PagedPlan;
  static Plan choose(const PagedView& p, int G, int n_q, int max_q, int64_t max_tokens, int n_splits) {
    return paged_kernels(p, G, n_q, max_q, max_tokens, n_splits);
  }
  static int64_t ws_bytes(const PagedView& p, int64_t rows, const Plan& k) { return paged_ws_bytes(p, rows, k); }
  // Workgroups of few rows for so many tiles of them.
  static double few_groups(const PagedView& p, const Plan& k, int64_t tiles) { return (double)tiles * p.H * k.few; }
};

template <class Kernels>
inline size_t attn_ws_bytes(const PagedView& p, int Hq, int n_q, int max_q, int max_tokens, int n_splits) {
  if (Hq < 1 || Hq % p.H != 0 || Hq / p.H > MUSTAFAR_PAGED_MAX_GROUP) return 0;
  if (n_q < 1 || max_q < 0 || max_tokens < 0 || n_splits > kMaxSplits || (int64_t)n_q * Hq >= kMaxRows) return 0;
  return (size_t)Kernels::ws_bytes(p, (int64_t)n_q * Hq, Kernels::choose(p, Hq / p.H, n_q, max_q, max_tokens, n_splits));
}

// Checks them and fills *a and *plan (not where n_q is 0: there is nothing to do).
template <class Kernels>
inline int attn_args(PagedAttnArgs* a, const void* q, int64_t q_stride, int n_q, int Hq, const PagedView& p, const void* cu,
                     int window, int sinks, float scale, void* out, int64_t out_stride, int max_q, int max_tokens, int n_splits,
                     void* ws, size_t ws_bytes, typename Kernels::Plan* plan) {
  if (Hq < 1 || Hq % p.H != 0 || n_q < 0 || max_q < 0 || max_tokens < 0 || window < 0 || sinks < 0) return MUSTAFAR_EINVAL;
  if (Hq / p.H > MUSTAFAR_PAGED_MAX_GROUP) return MUSTAFAR_EUNSUPPORTED;
  if (n_q == 0) return MUSTAFAR_OK;
  const int64_t row = (int64_t)Hq * p.d;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(cu, 4)) return MUSTAFAR_EINVAL;
  if (q_stride < row || out_stride < row || q_stride % 8 != 0 || out_stride % 8 != 0 || q_stride > (int64_t)1 << 31 ||
      out_stride > (int64_t)1 << 31)
    return MUSTAFAR_EINVAL;
  if ((int64_t)n_q * Hq >= kMaxRows) return MUSTAFAR_EINVAL;
  if (n_splits > kMaxSplits) return MUSTAFAR_EINVAL;
  const size_t need = attn_ws_bytes<Kernels>(p, Hq, n_q, max_q, max_tokens, n_splits);
  if (need > 0 && (!aligned(ws, 16) || ws_bytes < need)) return MUSTAFAR_EWORKSPACE;
  // (what the rows see: never more than the workspace was sized for)
  const int64_t seen = window > 0 ? (int64_t)window + max_q + sinks : max_tokens;
  const typename Kernels::Plan k = Kernels::choose(p, Hq / p.H, n_q, max_q, seen < max_tokens ? seen : max_tokens, n_splits);
  const int T = p.d / kTileChannels;
  const int64_t q_rows = (int64_t)n_q * Hq, few_rows = k.mixed ? (int64_t)p.B * p.H * kFewRows : q_rows;
  const int64_t few = k.mixed ? p.B : paged_tiles(p, Hq / p.H, n_q, kFewRows);
  const int64_t many = paged_tiles(p, Hq / p.H, n_q, chunk_rows(T));
  if (!launches(Kernels::few_groups(p, k, few), kWaveSize) || !launches((double)many * p.H * k.many, kWaveSize * chunk_waves(T)))
    return MUSTAFAR_EINVAL;
  if ((k.few > 1 && !launches((double)merge_groups(few_rows, T), kMergeThreads)) ||
      (k.many > 1 && !launches((double)merge_groups(q_rows, T), kMergeThreads)))
    return MUSTAFAR_EINVAL;
  *plan = k;
  a->p = p;
  a->few = k.few;
  a->many = k.many;
  a->mixed = k.mixed;
  a->few_rows = k.few_rows;
  a->by_entry = k.by_entry;
  a->ws = ws;
  a->q = (const uint16_t*)q;
  a->out = (uint16_t*)out;
  a->cu = (const int32_t*)cu;
  a->q_stride = q_stride;
  a->out_stride = out_stride;
  a->n_q = n_q;
  a->Hq = Hq;
  a->G = Hq / p.H;
  a->window = window;
  a->sinks = sinks;
  const double s = scale > 0.f ? (double)scale : 1.0 / sqrt((double)p.d);
  a->scale_log2 = (float)(s * 1.4426950408889634);
  return MUSTAFAR_OK;
}

}  // namespace mf
