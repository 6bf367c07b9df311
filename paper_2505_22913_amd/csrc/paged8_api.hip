// C ABI of the paged cache in 8 bits and of rotary positions (declared in include/mustafar.h):
// host-side checks, then the launches. Every check runs before any launch.
#include "paged_host.h"
#include "paged8.h"

using namespace mf;

namespace {

int check_pages8(const mustafar_pages8_t* c) {
  if (!c) return MUSTAFAR_EINVAL;
  const mustafar_pages_t* p = &c->pages;
  const int st = check_any_pages(p);
  if (st != MUSTAFAR_OK) return st;
  if (!is_code(p->type) || !is_16bit(c->type) || !c->k_scale || !c->v_scale) return MUSTAFAR_EINVAL;
  if (p->page_stride % 16 != 0 || p->head_stride % 16 != 0 || p->token_stride % 16 != 0) return MUSTAFAR_EINVAL;
  if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64) return MUSTAFAR_EINVAL;
  return c->block_tokens > p->page_tokens ? MUSTAFAR_EINVAL : MUSTAFAR_OK;
}

Paged8View view8_of(const mustafar_pages8_t* c) {
  Paged8View v;
  v.p = view_of(&c->pages);
  v.p.bf16 = c->type == MUSTAFAR_BF16;
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  v.int8 = c->pages.type == MUSTAFAR_INT8;
  v.log2_block = log2_of(c->block_tokens);
  return v;
}

bool stride_ok(int64_t stride, int64_t row) { return stride >= row && stride % 8 == 0 && stride <= (int64_t)1 << 31; }

}  // namespace

extern "C" {

int mustafar_paged8_init(mustafar_pages8_t* p, void* k, void* v, void* k_scale, void* v_scale, void* table, void* state,
                         void* free_pages, int B, int H, int d, int page_tokens, int n_pages, int max_pages, int type,
                         int code, int block_tokens, int64_t page_stride, int64_t head_stride, int64_t token_stride) {
  if (!p) return MUSTAFAR_EINVAL;
  mustafar_pages8_t t;
  t.pages = {k, v, (int32_t*)table, (int32_t*)state, (int32_t*)free_pages, B, H, d, page_tokens, n_pages, max_pages, code,
             page_stride, head_stride, token_stride};
  t.k_scale = (uint8_t*)k_scale;
  t.v_scale = (uint8_t*)v_scale;
  t.type = type;
  t.block_tokens = block_tokens;
  const int st = check_pages8(&t);
  if (st != MUSTAFAR_OK) return st;
  *p = t;
  return MUSTAFAR_OK;
}

int mustafar_paged8_write(const mustafar_pages8_t* p, const void* k_new, int64_t k_stride, const void* v_new,
                          int64_t v_stride, const void* cu, int n_new, void* stream) {
  const int st = check_pages8(p);
  if (st != MUSTAFAR_OK) return st;
  if (n_new < 0) return MUSTAFAR_EINVAL;
  if (n_new == 0) return MUSTAFAR_OK;
  const int64_t row = (int64_t)p->pages.H * p->pages.d;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(cu, 4)) return MUSTAFAR_EINVAL;
  if (!stride_ok(k_stride, row) || !stride_ok(v_stride, row)) return MUSTAFAR_EINVAL;
  const Paged8View c = view8_of(p);
  if (!launches((double)paged8_blocks(c.p, c.log2_block, n_new) * paged8_block_groups(c.p, c.log2_block), kWrite8Threads))
    return MUSTAFAR_EINVAL;
  return status_of(launch_paged8_write(c, (const uint16_t*)k_new, k_stride, (const uint16_t*)v_new, v_stride,
                                       (const int32_t*)cu, n_new, (hipStream_t)stream));
}

int mustafar_paged8_gather(const mustafar_pages8_t* p, const void* first, void* x_k, void* x_v, int n_max, void* stream) {
  const int st = check_pages8(p);
  if (st != MUSTAFAR_OK) return st;
  if (n_max < 0) return MUSTAFAR_EINVAL;
  if (n_max == 0) return MUSTAFAR_OK;
  if (!aligned(x_k, 16) || !aligned(x_v, 16) || (first && !aligned(first, 4))) return MUSTAFAR_EINVAL;
  const int64_t groups = ((int64_t)n_max * (p->pages.d / 8) + 255) / 256;  // of an entry and kv-head
  if (!launches((double)p->pages.B * p->pages.H * (double)groups, 256)) return MUSTAFAR_EINVAL;
  return status_of(launch_paged8_gather(view8_of(p), (const int32_t*)first, (uint16_t*)x_k, (uint16_t*)x_v, n_max,
                                        (hipStream_t)stream));
}

size_t mustafar_paged8_attn_workspace_bytes(const mustafar_pages8_t* p, int Hq, int n_q, int max_q, int max_tokens,
                                            int n_splits) {
  if (check_pages8(p) != MUSTAFAR_OK) return 0;
  return attn_ws_bytes<Kernels8>(view8_of(p).p, Hq, n_q, max_q, max_tokens, n_splits);
}

int mustafar_paged8_attn(const void* q, int64_t q_stride, int n_q, int Hq, const mustafar_pages8_t* p, const void* cu,
                         int window, int sinks, float scale, void* out, int64_t out_stride, int max_q, int max_tokens,
                         int n_splits, void* ws, size_t ws_bytes, void* stream) {
  const int st = check_pages8(p);
  if (st != MUSTAFAR_OK) return st;
  const Paged8View c = view8_of(p);
  Paged8AttnArgs a;
  Paged8Plan plan;
  const int what = attn_args<Kernels8>(&a, q, q_stride, n_q, Hq, c.p, cu, window, sinks, scale, out, out_stride, max_q, max_tokens,
                                       n_splits, ws, ws_bytes, &plan);
  if (what != MUSTAFAR_OK || n_q == 0) return what;
  a.k_scale = c.k_scale;
  a.v_scale = c.v_scale;
  a.int8 = c.int8;
  a.log2_block = c.log2_block;
  a.flat = plan.flat;
  a.budget = plan.budget;
  return status_of(launch_paged8_attn(a, (hipStream_t)stream));
}

int mustafar_rope_rates(double* rates, int rot, double base, int scaling, double factor, double original_len,
                        double low_turns, double high_turns) {
  if (!rates || rot < 2 || rot > MUSTAFAR_ROPE_MAX_D || rot % 2 != 0) return MUSTAFAR_EINVAL;
  if (!isfinite(base) || base <= 0 || scaling < MUSTAFAR_ROPE_PLAIN || scaling > MUSTAFAR_ROPE_TURNS) return MUSTAFAR_EINVAL;
  if (scaling == MUSTAFAR_ROPE_PLAIN) factor = 1;
  if (!isfinite(factor) || factor <= 0) return MUSTAFAR_EINVAL;
  double slower = 1;  // factor's part of the rates is slower^(-2 i / (rot - 2)) where the enlarged base is no normal number
  if (scaling == MUSTAFAR_ROPE_BASE) {
    if (rot == 2) return MUSTAFAR_EINVAL;
    const double enlarged = base * pow(factor, (double)rot / (rot - 2));
    if (isnormal(enlarged)) base = enlarged;
    else slower = factor;
    factor = 1;
  }
  const bool turns = scaling == MUSTAFAR_ROPE_TURNS;
  if (turns && (!isfinite(original_len) || original_len <= 0 || !isfinite(low_turns) || !isfinite(high_turns) ||
                low_turns >= high_turns))
    return MUSTAFAR_EINVAL;
  double r[MUSTAFAR_ROPE_MAX_D / 2];
  for (int i = 0; i < rot / 2; ++i) {
    r[i] = pow(base, -2.0 * i / rot);
    if (slower != 1) r[i] *= pow(slower, -2.0 * i / (rot - 2));
    double keep = 0;
    if (turns) {
      keep = (original_len * r[i] / (2 * M_PI) - low_turns) / (high_turns - low_turns);
      keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
    }
    r[i] *= keep + (1 - keep) / factor;
    if (!isfinite(r[i])) return MUSTAFAR_EINVAL;
  }
  for (int i = 0; i < rot / 2; ++i) rates[i] = r[i];
  return MUSTAFAR_OK;
}

int mustafar_rope(const mustafar_rotation_t* r, const void* q, int64_t q_stride, int Hq, const void* k, int64_t k_stride,
                  int H, int d, int n, int type, const void* positions, const mustafar_pages_t* p, const void* cu,
                  int inverse, void* out_q, int64_t out_q_stride, void* out_k, int64_t out_k_stride, void* stream) {
  if (!r || !aligned(r->rates, 8) || r->rot < 2 || r->rot % 2 != 0 || r->rot > d || d < 8 || d % 8 != 0 ||
      d > MUSTAFAR_ROPE_MAX_D)
    return MUSTAFAR_EINVAL;
  if (r->layout != MUSTAFAR_ROPE_HALF && r->layout != MUSTAFAR_ROPE_INTERLEAVED) return MUSTAFAR_EINVAL;
  if (!is_16bit(type) || n < 0 || Hq < 0 || H < 0 || Hq > kMaxRopeHeads || H > kMaxRopeHeads || Hq + H == 0)
    return MUSTAFAR_EINVAL;
  if (n > 0 && (positions ? p || cu || !aligned(positions, 4) : !p || !aligned(cu, 4))) return MUSTAFAR_EINVAL;
  if (p && check_any_pages(p) != MUSTAFAR_OK) return MUSTAFAR_EINVAL;
  auto side_ok = [&](const void* x, int64_t stride, int heads, const void* out, int64_t out_stride) {
    if (heads == 0) return !x && !out;
    const int64_t row = (int64_t)heads * d;
    return stride_ok(stride, row) && stride_ok(out_stride, row) && (x != out || stride == out_stride) &&
           (n == 0 || (aligned(x, 16) && aligned(out, 16)));
  };
  if (!side_ok(q, q_stride, Hq, out_q, out_q_stride) || !side_ok(k, k_stride, H, out_k, out_k_stride)) return MUSTAFAR_EINVAL;
  if (n == 0) return MUSTAFAR_OK;
  RopeArgs a;
  a.rates = r->rates;
  a.rot = r->rot;
  a.layout = r->layout;
  a.magnitude = r->magnitude;
  a.bf16 = type == MUSTAFAR_BF16;
  a.inverse = inverse != 0;
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.out_q = (uint16_t*)out_q;
  a.out_k = (uint16_t*)out_k;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.out_q_stride = out_q_stride;
  a.out_k_stride = out_k_stride;
  a.Hq = Hq;
  a.H = H;
  a.d = d;
  a.n = n;
  a.positions = (const int32_t*)positions;
  a.cu = (const int32_t*)cu;
  a.state = p ? p->state : nullptr;
  a.B = p ? p->B : 0;
  a.most = p ? (int64_t)p->max_pages * p->page_tokens : 0;
  const RopePlan plan = rope_plan(a);
  if (!launches((double)plan.groups, kRopeThreads)) return MUSTAFAR_EINVAL;
  return status_of(launch_rope(a, plan, (hipStream_t)stream));
}

}  // extern "C"
