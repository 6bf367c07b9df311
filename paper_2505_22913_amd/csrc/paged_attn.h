// What the attention kernels over pages share (paged_attn.hip: 16-bit pages, paged8_attn.hip: pages
// of 8-bit codes): the rows of a launch, the tiles that they see, a row by itself, ranges' results.
#pragma once

#include "mf_device.h"
#include "paged.h"

namespace mf {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------
// The two 16-bit types.
// ------------------------------------------------------------------------------------------
template <bool BF16>
__device__ __forceinline__ float to_float(uint32_t bits) {
  if constexpr (BF16) return __builtin_bit_cast(float, bits << 16);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// Two values rounded to nearest even, the first in the low half.
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const f32x2 v = {x, y};
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2_t));
}

// c + the sum of a pair.
template <bool BF16>
__device__ __forceinline__ float add_pair(uint32_t pair, float c) {
  if constexpr (BF16) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), (bf16x2){(__bf16)1.f, (__bf16)1.f}, c, false);
  } else {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2_t, pair), (half2_t){(_Float16)1.f, (_Float16)1.f}, c, false);
  }
}

// D[32][32] = A[32][16] B[16][32] + C: lane l holds A's row and B's column l % 32 at k = 8 (l / 32) + i,
// and column l % 32 of the result at rows 8 (r / 4) + 4 (l / 32) + r % 4.
template <bool BF16>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

template <bool BF16>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

// ------------------------------------------------------------------------------------------
// Rows, tokens, tiles.
// ------------------------------------------------------------------------------------------
// The rows of a request are its new tokens times the G query heads of a kv-head, so that a kv-head's keys are read once for all
// of them; a workgroup takes BM consecutive ones. Every workgroup counts the requests' tiles for itself, so that those without
// work are the launch's last ones: spread over it, a third of them made 16 requests of 512 rows (256 workgroups for 256 CUs)
// take two turns, 76 us for 40.
struct RowTile {
  int b, row0, rows;  // request, first row, rows of the request (row0 >= rows: nothing to do)
  int base;           // position of the request's first new token
  int tok0;           // its row in q
};

__device__ __forceinline__ RowTile rows_at(const PagedAttnArgs& a, int b, int cu, int cu_next, int len) {
  RowTile r;
  r.b = b;
  r.row0 = 0;
  r.tok0 = cu;
  const int nq = min(cu_next, a.n_q) - cu;
  r.rows = nq * a.G;
  r.base = (int)min((int64_t)max(len, 0), (int64_t)a.p.max_pages << a.p.log2_page) - nq;
  return r;
}

__device__ __forceinline__ RowTile rows_of(const PagedAttnArgs& a, int b) {
  const int cu = a.cu[b], next = a.cu[b + 1], len = a.p.state[b];
  return rows_at(a, b, __builtin_amdgcn_readfirstlane(cu), __builtin_amdgcn_readfirstlane(next), __builtin_amdgcn_readfirstlane(len));
}

// The last request that `begins` (its first row, its number) is true of, its rows [cu, next) and its length: of up to 64 requests by one
// round of loads, else by two and its own.
struct Request {
  int b, cu, next, len;
};
template <class Begins>
__device__ __forceinline__ Request last_request(const int32_t* starts, const int32_t* lens, int B, Begins begins) {
  const int lane = (int)lane_id();
  if (B <= kWave) {
    const int b = min(lane, B - 1), cu = starts[b], next = starts[b + 1], len = lens[b];
    const int at = 63 - __builtin_clzll(ballot(lane < B && begins(cu, b)) | 1);
    return {at, __builtin_amdgcn_readlane(cu, at), __builtin_amdgcn_readlane(next, at), __builtin_amdgcn_readlane(len, at)};
  }
  const int stride = (B + kWave - 1) / kWave;
  int b = min(lane * stride, B - 1);
  b = (63 - __builtin_clzll(ballot(lane * stride < B && begins(starts[b], b)) | 1)) * stride;
  const int in = min(b + lane, B - 1);
  const uint64_t below = ballot(lane < stride && b + lane < B && begins(starts[in], in));
  b = __builtin_amdgcn_readfirstlane(b + 63 - (int)__builtin_clzll(below | 1));
  const int cu = starts[b], next = starts[b + 1], len = lens[b];
  return {b, __builtin_amdgcn_readfirstlane(cu), __builtin_amdgcn_readfirstlane(next), __builtin_amdgcn_readfirstlane(len)};
}
// The request that holds row t of a step.
__device__ __forceinline__ Request request_at(const int32_t* starts, const int32_t* lens, int B, int t) {
  return last_request(starts, lens, B, [&](int cu, int) { return cu <= t; });
}
__device__ __forceinline__ RowTile request_of(const PagedAttnArgs& a, int t) {
  const Request r = request_at(a.cu, a.p.state, a.p.B, t);
  return rows_at(a, r.b, r.cu, r.next, r.len);
}

// Tile `tile` of the launch: all requests' tiles (with `many`: of the requests of more than kFewRows rows) from the last one to the
// first, so that a request's longest come first. row0 >= rows: there are not so many.
template <int BM>
__device__ __forceinline__ RowTile row_tile(const PagedAttnArgs& a, int tile, bool many) {
  const int B = a.p.B, lane = (int)lane_id(), stride = (B + kWave - 1) / kWave;
  auto tiles = [&](int b) {
    const int rows = (min(a.cu[b + 1], a.n_q) - a.cu[b]) * a.G;
    return rows <= (many ? kFewRows : 0) ? 0u : (uint32_t)(rows + BM - 1) / BM;
  };
  // Lane i: the tiles of requests stride * i ..; then the requests of the lane that has the wanted one.
  uint32_t n = 0;
  for (int b = lane * stride; b < min((lane + 1) * stride, B); ++b) n += tiles(b);
  uint32_t incl = wave_incl_scan(n);
  const uint32_t total = __builtin_amdgcn_readlane(incl, kWave - 1);
  RowTile r;
  if ((uint32_t)tile >= total) {
    r.row0 = r.rows = 0;
    return r;
  }
  uint32_t want = total - 1 - (uint32_t)tile;
  int at = __builtin_popcountll(ballot(incl <= want));
  want -= __builtin_amdgcn_readlane(incl - n, at);
  if (stride > 1) {
    at *= stride;
    n = lane < stride && at + lane < B ? tiles(at + lane) : 0u;
    incl = wave_incl_scan(n);
    const int x = __builtin_popcountll(ballot(incl <= want));
    want -= __builtin_amdgcn_readlane(incl - n, x);
    at += x;
  }
  r = rows_of(a, at);
  r.row0 = (int)want * BM;
  return r;
}

// The newest token that a window ending at pos leaves out (-1: none; the difference may leave 32 bits).
__device__ __forceinline__ int before(int pos, int window) { return (int)max((int64_t)pos - window, (int64_t)-1); }

// The tokens that rows at positions [pos0, pos1] see between them, [0, sinks) and [lo, hi], in tiles of BN:
// tile i of the list starts at token start(i).
struct TileList {
  int sinks, lo, hi;
  int first, n_first;  // the tile of lo (or 0), and how many of the sinks' come before it
  int n;
  __device__ __forceinline__ TileList(int pos0, int pos1, int window, int n_sinks, int BN) {
    hi = pos1;
    lo = window > 0 ? before(pos0, window) + 1 : 0;
    sinks = min(n_sinks, lo);
    n_first = (sinks + BN - 1) / BN;
    first = lo / BN;
    if (n_first >= first) {
      n_first = 0;
      if (sinks > 0) first = 0;
    }
    n = hi < 0 ? 0 : n_first + hi / BN - first + 1;
  }
  // Tiles of the list that start at or before token j.
  __device__ __forceinline__ int count_to(int j, int BN) const {
    if (j < 0) return 0;
    return j / BN < first ? min(n_first, j / BN + 1) : n_first + j / BN - first + 1;
  }
  __device__ __forceinline__ int start(int i, int BN) const { return (i < n_first ? i : first + i - n_first) * BN; }
};

__device__ __forceinline__ bool sees(int pos, int j, int window, int n_sinks) {
  return j <= pos && (window == 0 || j > pos - window || j < n_sinks);
}

// ------------------------------------------------------------------------------------------
// A row by itself, one wave: every product in fp32 on the vector units, and nothing of a token that
// the row does not see. The kernels below come here with the rows of a wave whose result is not
// finite: their matrix products take whole tiles, so that a value that is not finite reaches
// the rows that do not see it (0 times infinity). Latency bounds it, a row of 4096 tokens takes more than a millisecond: a
// prompt of 4096 with 32 heads, 170 us, takes 29 to 31 ms where every row of one head sees an infinity, 46 to 51 where those of all do,
// 42 to 44 where only the last row does.
// ------------------------------------------------------------------------------------------
// The least weight of a visible token: an infinite value that one sees stays infinite
// where its probability is under fp32's range (0 times infinity would be NaN).
constexpr float kLeast = 0x1p-120f;
__device__ __forceinline__ float at_least(float x) { return x < kLeast ? kLeast : x; }  // (NaN stays)

template <int T>
struct RowState {
  float m, l, o[T];  // o: channels lane + 64 c
};

// Sums of bf16 values leave fp32 where their mean, the output, does not. So weights are at most 2^-one_below() here, 1 over
// more than twice the tokens' number, and a sum is no larger than half the largest value. (It costs the smallest values precision:
// products under 2^-126 are multiples of 2^-149, so that the output of n tokens is off by up to 4 n^2 2^-150.)
template <bool BF16>
__device__ __forceinline__ float one_below(TileList tl, int BN) {
  return BF16 ? (float)(64 - __builtin_clz(tl.n | 1) - __builtin_clz(BN)) : 0.f;
}

// A token's key and value in 16-bit pages; `held` is what a lane keeps of its token, `passed` what one lane gets of another's.
template <bool BF16>
struct Pages16 {
  struct Held { int64_t at; };
  const PagedView& p;
  __device__ __forceinline__ Held held(int page, int h, int place) const {
    return {(int64_t)page * p.page_stride + (int64_t)h * p.head_stride + (int64_t)place * p.token_stride};
  }
  __device__ __forceinline__ float key(const Held& t, int c) const { return to_float<BF16>(p.k[t.at + c]); }
  __device__ __forceinline__ Held passed(const Held& t, int lane) const { return {(int64_t)__shfl(t.at, lane, kWave)}; }
  __device__ __forceinline__ float value(const Held& t, int c) const { return to_float<BF16>(p.v[t.at + c]); }
};

template <int T, bool BF16, class Pages>
__device__ __forceinline__ RowState<T> one_row(const PagedAttnArgs& a, const Pages& pages, int b, int h, const uint16_t* q, int pos,
                                            TileList tl, int t0, int t1, int BN) {
  constexpr int d = kTile * T;
  const PagedView& p = a.p;
  const int lane = (int)lane_id();
  const float below = one_below<BF16>(tl, BN);
  RowState<T> s;
  s.m = -INFINITY;
  s.l = 0.f;
  for (int c = 0; c < T; ++c) s.o[c] = 0.f;
  for (int t = t0; t < t1; ++t) {
    const int j0 = tl.start(t, BN), j = j0 + lane;
    const bool seen = lane < BN && j <= tl.hi && sees(pos, j, a.window, a.sinks);
    typename Pages::Held at = {};
    float x = -INFINITY;
    if (seen) {
      int page = p.table[(int64_t)b * p.max_pages + (j >> p.log2_page)];
      if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
      at = pages.held(page, h, j & ((1 << p.log2_page) - 1));
      x = 0.f;
      for (int c = 0; c < d; ++c) x = fmaf(to_float<BF16>(q[c]), pages.key(at, c), x);
    }
    const float mnew = fmaxf(s.m, wave_max(x));
    const float alpha = s.m == -INFINITY ? 1.f : at_least(__builtin_amdgcn_exp2f((s.m - mnew) * a.scale_log2));
    const float w = x == -INFINITY ? 0.f : at_least(__builtin_amdgcn_exp2f(fmaf(x - mnew, a.scale_log2, -below)));
    s.m = mnew;
    s.l = fmaf(s.l, alpha, wave_sum(w));
    for (int c = 0; c < T; ++c) s.o[c] *= alpha;
    for (uint64_t left = ballot(seen); left; left &= left - 1) {
      const int i = __builtin_ctzll(left);
      const float wi = __shfl(w, i, kWave);
      const typename Pages::Held ai = pages.passed(at, i);
      for (int c = 0; c < T; ++c) s.o[c] = fmaf(wi, pages.value(ai, kTile * c + lane), s.o[c]);
    }
  }
  return s;
}

// ------------------------------------------------------------------------------------------
// Results: the rounded output, or one range's share of it for k_paged_merge: the log2 of what its weights are multiples of
// (-inf if it has none), their sum (-1 for a row that sees nothing at all) and the weighted values.
// ------------------------------------------------------------------------------------------
struct PartOut {
  float2* ml;  // [n_splits][rows]
  float* o;    // [n_splits][rows][d]
  int64_t rows;
  int by_entry;
  int n_splits;
};

// Row r of a request and kv-head among a range's.
__device__ __forceinline__ int64_t part_row(const PagedAttnArgs& a, const PartOut& part, const RowTile& rt, int h, int r) {
  if (part.by_entry) return ((int64_t)rt.b * a.p.H + h) * kFewRows + r;
  const int tok = r / a.G;
  return (int64_t)(rt.tok0 + tok) * a.Hq + h * a.G + r - tok * a.G;
}

// result_at(r): where the range's results of row r of the request go, if there are several.
template <int T, bool BF16, class Pages, class At>
__device__ __forceinline__ void redo_rows(const PagedAttnArgs& a, const Pages& pages, const PartOut& part, const RowTile& rt, int h, int first_row,
                                       int n_rows, TileList tl, int t0, int t1, At result_at, int BN) {
  constexpr int d = kTile * T;
  const int lane = (int)lane_id();
  for (int r = first_row; r < min(first_row + n_rows, rt.rows); ++r) {
    const int tok = r / a.G, hq = h * a.G + (r - tok * a.G), t = rt.tok0 + tok, pos = rt.base + tok;
    const RowState<T> s = one_row<T, BF16>(a, pages, rt.b, h, a.q + t * a.q_stride + hq * d, pos, tl, t0, t1, BN);
    if (part.n_splits > 1) {
      const int64_t row = result_at(r);
      // (what the maximum's rounding leaves goes into the sums: other ranges' are multiples of 2^m with theirs. Beyond 2^27 scores
      // of fp32 differ by more than 2^8 or not at all. bf16: a factor of up to 2^8 is room that m gives the sums.)
      const float below = one_below<BF16>(tl, BN), more = BF16 && fabsf(s.m * a.scale_log2) >= 0x1p24f ? 8.f : 0.f;
      const float m = fmaf(s.m, a.scale_log2, below + more), left = fmaf(s.m, a.scale_log2, -m) + below;
      const float f = __builtin_amdgcn_exp2f(fminf(fmaxf(left, -more - 8.f), -more + 8.f));
      if (lane == 0) part.ml[row] = make_float2(m, pos < 0 ? -1.f : s.l * f);
      for (int c = 0; c < T; ++c) part.o[row * d + kTile * c + lane] = s.o[c] * f;
    } else {
      for (int c = 0; c < T; ++c)
        a.out[t * a.out_stride + hq * d + kTile * c + lane] = (uint16_t)pack2<BF16>(pos < 0 ? 0.f : s.o[c] / s.l, 0.f);
    }
  }
}

// ------------------------------------------------------------------------------------------
// The n_splits ranges of a row together, into row t and head hq of a.out: range s of it lies at row + s * rows of ml and o.
// ------------------------------------------------------------------------------------------
constexpr int kMergeAhead = 8, kMergeWideRows = 512;

template <int T, bool BF16, int OF, bool WIDE>
__device__ __forceinline__ void merge_row(const PagedAttnArgs& a, const float2* ml, const float* o_of, int64_t rows, int n_splits,
                                          int64_t row, int t, int hq) {
  constexpr int d = kTile * T, L = 16 * T, S = kMergeThreads / L;
  constexpr int kStep = WIDE ? S : 1, kAhead = kMergeAhead < OF / kStep ? kMergeAhead : OF / kStep;
  static_assert(OF % (kStep * kAhead) == 0, "the ranges under way are of one round of weights");
  const int lane = (int)lane_id(), stream = (int)threadIdx.x / L, sub = (int)threadIdx.x % L;
  const int first = WIDE ? stream : 0, at = lane % OF;
  f32x4 x[kAhead], o = {};
  auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (s0 + kStep * k < n_splits) x[k] = *reinterpret_cast<const f32x4*>(o_of + ((s0 + kStep * k) * rows + row) * d + 4 * sub);
  };
  load(first);
  // (bf16: ranges' outputs may be as large as fp32 holds; times less than 1 part in their number, so is their sum)
  const float down = BF16 ? __builtin_bit_cast(float, (uint32_t)(95 + __builtin_clz(n_splits)) << 23) : 1.f;
  float M = -INFINITY, l = 0.f;
  for (int s = at; s < n_splits; s += OF) M = fmaxf(M, ml[s * rows + row].x);
#pragma unroll
  for (int k = 1; k < OF; k *= 2) M = fmaxf(M, __shfl_xor(M, k, kWave));
  uint64_t nothing = 0;
  for (int s0 = 0; s0 < n_splits; s0 += OF) {
    // lane i of those: the weight of range s0 + i, 0 for one without any (its output is not looked at)
    float2 of = make_float2(-INFINITY, 0.f);
    if (s0 + at < n_splits) of = ml[(s0 + at) * rows + row];
    const float w = of.x != -INFINITY || of.y != 0.f ? at_least(__builtin_amdgcn_exp2f(of.x - M)) * down : 0.f;
    if (w != 0.f) l = fmaf(of.y, w, l);
    nothing |= ballot(of.y < 0.f);
    const int end = min(s0 + OF, n_splits);
    for (int s = s0; s < end; s += kStep * kAhead) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int sk = s + first + kStep * k;
        if (OF == kMergeAhead && sk >= end) break;
        const float wk = __shfl(w, (lane & -OF) | ((sk - s0) % OF), kWave);
        if (sk < end && wk != 0.f)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = fmaf(x[k][e], wk, o[e]);
      }
      load(s + first + kStep * kAhead);
    }
  }
#pragma unroll
  for (int k = 1; k < OF; k *= 2) l += __shfl_xor(l, k, kWave);
  const bool zero = (nothing >> (lane & -OF) & (~0ull >> (kWave - OF))) != 0;
  if constexpr (WIDE) {
    __shared__ f32x4 sums[kMergeThreads / kWave][L];
#pragma unroll
    for (int k = L; k < kWave; k *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], k, kWave);
    if (lane < L) sums[threadIdx.x / kWave][lane] = o;
    __syncthreads();
    if (threadIdx.x >= L) return;
    o = sums[0][sub];
#pragma unroll
    for (int w = 1; w < kMergeThreads / kWave; ++w) o += sums[w][sub];
  }
  u32x2 y = {};
  if (!zero) y = (u32x2){pack2<BF16>(o[0] / l, o[1] / l), pack2<BF16>(o[2] / l, o[3] / l)};
  *reinterpret_cast<u32x2*>(a.out + t * a.out_stride + hq * d + 4 * sub) = y;
}

// ------------------------------------------------------------------------------------------
// Tiles in LDS, and the softmax's reference.
// ------------------------------------------------------------------------------------------
template <int T>
constexpr int chunk_tile() { return T == 4 ? 32 : 64; }

// A probability is 2^kBias at the reference, which follows the largest score once that is more than 2^kSlack above it:
// at most 2^15 (inside fp16), and fp16 keeps those down to 2^-31 of the reference. It is exp2(score * scale +
// shift) with shift = kBias - reference * scale rounded: one shift for all weights of a row, so its rounding is a
// factor of them all: under kFar at most 2 (fp16, whose small weights it must not lose) and 2^8 (bf16, for the
// least weight of k_paged_merge's ranges). Rows with larger shifts are done by themselves.
constexpr float kBias = 7.f, kSlack = 8.f;
template <bool BF16>
constexpr float kFar = BF16 ? 0x1p28f : 0x1p25f;

// 16-byte pieces of a row are stored at their place XOR these, so that the lanes of a read (K: one piece of
// many rows; V: 32 or 64 bytes of four rows) find them in different banks.
template <int T>
__device__ __forceinline__ uint32_t swizzle_k(uint32_t row) { return T == 1 ? row % 8 : row % 16; }
template <int T>
__device__ __forceinline__ uint32_t swizzle_v(uint32_t row) {
  return T == 1 ? 2 * (row & 3) : ((row & 1) ? 6u : 0u) ^ ((row & 2) ? 10u : 0u);
}

// 16 bytes a lane from base + offset to LDS at dst + 16 lane; wait_loads() waits for them. (Inline: behind the builtin the
// compiler waits for every such load before the next transposing LDS read of any address. The load has no register
// output; m0, its LDS address, is put back. Five cycles lie between a base that the vector units wrote and its use.)
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t dst) {
  const uint64_t at = (uint64_t)base;  // (uniform; said so, whatever the compiler makes of how it came about)
  const uint64_t sbase = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)) << 32 |
                         (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at);
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(__builtin_amdgcn_readfirstlane((int)dst)), "v"(offset), "s"(sbase) : "memory");
}
template <int LEFT>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LEFT) : "memory"); }

template <typename V>
__device__ __forceinline__ V lds_load(uint32_t byte_addr) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V*>(byte_addr);
}
// Four tokens of one channel: the 16 lanes of a group address 4 x 16 elements, and each gets a column.
__device__ __forceinline__ u32x2 lds_load_tr(uint32_t byte_addr) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       reinterpret_cast<__attribute__((address_space(3))) s16x4*>(byte_addr)));
}

// Largest over the two lanes of a row.
__device__ __forceinline__ float max_halves(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

template <int NK>
__device__ __forceinline__ float max_of(const f32x16 (&s)[NK]) {
  float top = s[0][0];
#pragma unroll
  for (int n = 0; n < NK; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][r]);
  return top;
}

// Joins the ranges of the kernel that has the requests of few rows, or of the other, into a.out (paged_attn.hip).
hipError_t launch_paged_merge(const PagedAttnArgs& a, const PartOut& part, bool of_few, hipStream_t s);

}  // namespace mf
