// Causal attention of the new tokens of every request over its pages (gfx950), with an
// optional sliding window and first tokens that stay visible.
#include <type_traits>

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

// The request that holds row t of q: of up to 64 requests by one round of loads, else by two and its own.
__device__ __forceinline__ RowTile request_of(const PagedAttnArgs& a, int t) {
  const int B = a.p.B, lane = (int)lane_id();
  if (B <= kWave) {
    const int b = min(lane, B - 1), cu = a.cu[b], next = a.cu[b + 1], len = a.p.state[b];
    const int at = 63 - __builtin_clzll(ballot(lane < B && cu <= t) | 1);
    return rows_at(a, at, __builtin_amdgcn_readlane(cu, at), __builtin_amdgcn_readlane(next, at), __builtin_amdgcn_readlane(len, at));
  }
  const int stride = (B + kWave - 1) / kWave;
  const int b = (63 - __builtin_clzll(ballot(lane * stride < B && a.cu[min(lane * stride, B - 1)] <= t) | 1)) * stride;
  const uint64_t below = ballot(lane < stride && b + lane < B && a.cu[min(b + lane, B - 1)] <= t);
  return rows_of(a, __builtin_amdgcn_readfirstlane(b + 63 - (int)__builtin_clzll(below | 1)));
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
// prompt of 4096 with 32 heads, 170 us, takes 29 ms where every row of one head sees an infinity, 46 where those of all do, 42
// where only the last row does.
// ------------------------------------------------------------------------------------------
// The least weight of a visible token: an infinite value that one sees stays infinite
// where its probability is under fp32's range (0 times infinity would be NaN).
constexpr float kLeast = 0x1p-120f;
__device__ __forceinline__ float at_least(float x) { return x < kLeast ? kLeast : x; }  // (NaN stays)

template <int T>
struct RowState {
  float m, l, o[T];  // o: channels lane + 64 c
};

template <int T, bool BF16>
__device__ __forceinline__ RowState<T> one_row(const PagedAttnArgs& a, int b, int h, const uint16_t* q, int pos, TileList tl,
                                            int t0, int t1, int BN) {
  constexpr int d = kTile * T;
  const PagedView& p = a.p;
  const int lane = (int)lane_id();
  RowState<T> s;
  s.m = -INFINITY;
  s.l = 0.f;
  for (int c = 0; c < T; ++c) s.o[c] = 0.f;
  for (int t = t0; t < t1; ++t) {
    const int j0 = tl.start(t, BN), j = j0 + lane;
    const bool seen = lane < BN && j <= tl.hi && sees(pos, j, a.window, a.sinks);
    int64_t at = 0;
    float x = -INFINITY;
    if (seen) {
      int page = p.table[(int64_t)b * p.max_pages + (j >> p.log2_page)];
      if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
      at = (int64_t)page * p.page_stride + (int64_t)h * p.head_stride +
           (int64_t)(j & ((1 << p.log2_page) - 1)) * p.token_stride;
      x = 0.f;
      for (int c = 0; c < d; ++c) x = fmaf(to_float<BF16>(q[c]), to_float<BF16>(p.k[at + c]), x);
    }
    const float mnew = fmaxf(s.m, wave_max(x));
    const float alpha = s.m == -INFINITY ? 1.f : at_least(__builtin_amdgcn_exp2f((s.m - mnew) * a.scale_log2));
    const float w = x == -INFINITY ? 0.f : at_least(__builtin_amdgcn_exp2f((x - mnew) * a.scale_log2));
    s.m = mnew;
    s.l = fmaf(s.l, alpha, wave_sum(w));
    for (int c = 0; c < T; ++c) s.o[c] *= alpha;
    for (uint64_t left = ballot(seen); left; left &= left - 1) {
      const int i = __builtin_ctzll(left);
      const float wi = __shfl(w, i, kWave);
      const int64_t ai = __shfl(at, i, kWave);
      for (int c = 0; c < T; ++c) s.o[c] = fmaf(wi, to_float<BF16>(p.v[ai + kTile * c + lane]), s.o[c]);
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

template <int T, bool BF16>
__device__ __forceinline__ void redo_rows(const PagedAttnArgs& a, const PartOut& part, const RowTile& rt, int h, int first_row,
                                       int n_rows, TileList tl, int t0, int t1, int split, int BN) {
  constexpr int d = kTile * T;
  const int lane = (int)lane_id();
  for (int r = first_row; r < min(first_row + n_rows, rt.rows); ++r) {
    const int tok = r / a.G, hq = h * a.G + (r - tok * a.G), t = rt.tok0 + tok, pos = rt.base + tok;
    const RowState<T> s = one_row<T, BF16>(a, rt.b, h, a.q + t * a.q_stride + hq * d, pos, tl, t0, t1, BN);
    if (part.n_splits > 1) {
      const int64_t row = split * part.rows + part_row(a, part, rt, h, r);
      // (what the maximum's rounding leaves goes into the sums: other ranges' are multiples of 2^m with theirs. Beyond 2^27 scores
      // of fp32 differ by more than 2^8 or not at all.)
      const float m = s.m * a.scale_log2, f = __builtin_amdgcn_exp2f(fminf(fmaxf(fmaf(s.m, a.scale_log2, -m), -8.f), 8.f));
      if (lane == 0) part.ml[row] = make_float2(m, pos < 0 ? -1.f : s.l * f);
      for (int c = 0; c < T; ++c) part.o[row * d + kTile * c + lane] = s.o[c] * f;
    } else {
      for (int c = 0; c < T; ++c)
        a.out[t * a.out_stride + hq * d + kTile * c + lane] = (uint16_t)pack2<BF16>(pos < 0 ? 0.f : s.o[c] / s.l, 0.f);
    }
  }
}

// ------------------------------------------------------------------------------------------
// k_paged_chunk: 32 rows a wave, 8 waves a workgroup (4 at d = 256), tiles of 64 tokens (32).
//
// Both products have the rows as columns: S^T = K Q^T leaves a lane with scores of one row (column l % 32),
// so the softmax's shift and sum are per lane (two lanes hold a row's tokens), and its 8-token groups,
// rounded to the type, are the B operand of O^T = V^T P^T as they lie; V^T comes out of LDS transposed.
//
// Step t is X, the products of tile t + 1's scores, then the probabilities of tile t, then Y, the products with its values, then
// the maximum of tile t + 1's scores; the products are fenced one by one, so that the reads of their operands stay ahead of them.
// One barrier a step. Tiles are staged kDepth steps ahead (pair t: the keys of tile t + 1 and the values of tile t) and arrive one
// step before they are needed, so that the first operands of a step are read before its barrier; they go where the step
// before has read.
//
// The matrix units and the vector units bound it, hardly ever at once: of 4 prompts of 4096 tokens with 32 heads at d = 128 (550 GFLOP
// of visible pairs), 535 to 570 us from one card to the next (1.03 to 0.96 PFLOP/s, where a product of 8192^3 reaches 1.23 to
// 1.19), the first are busy for half of the cycles and the second for 45%, at the 1.9 GHz of 2.4 that the card's power leaves
// them; LDS has no conflicts. The same with d = 64: 358 us, 0.77 PFLOP/s. One prompt of 4096 with 16 heads at d = 256: 155 to 167 us,
// 0.89 to 0.82 PFLOP/s. A workgroup alone on its CU (128 KB of LDS) starts
// and ends in 9 us and takes 1.7 a tile. Tried at the first size: the probabilities between the products of X and Y, 566 us for 548; Y
// before X, so that one buffer of scores will do, 573 for 545, with four of the eight waves half a step later 596; 64
// rows a wave and one wave a SIMD, 694 for 592; two workgroups of 4 waves a CU and tiles of 32, 586 for 543; a tile's loads all at
// once, 628 for 602; other wave priorities, 4 and 6 operands ahead: no gain.
// ------------------------------------------------------------------------------------------
template <int T>
constexpr int chunk_tile() { return T == 4 ? 32 : 64; }
constexpr int kDepth = 3, kRing = kDepth + 1;

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

template <int T, bool BF16>
__global__ __launch_bounds__(chunk_waves(T) * kWave, T == 4 ? 1 : 2) void k_paged_chunk(PagedAttnArgs a, PartOut part) {
  constexpr int NW = chunk_waves(T), BM = 32 * NW;
  constexpr int d = kTile * T, BN = chunk_tile<T>(), NK = BN / 32, NC = d / 16, ND = d / 32;
  constexpr uint32_t kRow = 2 * d, kBuf = BN * kRow;  // bytes
  constexpr int kWaveRows = BN / NW, kRowsPerLoad = 1024 / (2 * d), kLoads = kWaveRows / kRowsPerLoad;
  static_assert(kLoads * kRowsPerLoad == kWaveRows && 16 % kWaveRows == 0, "a wave's rows");
  __shared__ __align__(1024) unsigned char smem[(2 * kRing) * kBuf];  // buffers of keys, of values
  const PagedView& p = a.p;
  const int h = blockIdx.x % p.H, split = (blockIdx.x / p.H) % part.n_splits, tile = (int)(blockIdx.x / (p.H * part.n_splits));
  const RowTile rt = row_tile<BM>(a, tile, a.mixed != 0);
  if (rt.row0 >= rt.rows) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const uint32_t lane = lane_id(), r32 = lane % 32, half = lane / 32;
  const int wrow = rt.row0 + 32 * wave;  // the wave's first row
  const TileList tl(rt.base + rt.row0 / a.G, rt.base + (min(rt.row0 + BM, rt.rows) - 1) / a.G, a.window, a.sinks, BN);
  const int t0 = (int)((int64_t)tl.n * split / part.n_splits);
  const int n = (int)((int64_t)tl.n * (split + 1) / part.n_splits) - t0;  // tiles of the workgroup
  // The wave's rows' positions, and its tiles: those behind its last position are the others'.
  const int pos0 = rt.base + min(wrow, rt.rows - 1) / a.G, pos1 = rt.base + min(wrow + 31, rt.rows - 1) / a.G;
  const int mine = wrow >= rt.rows || pos1 < 0 ? 0 : min(n, max(tl.count_to(pos1, BN) - t0, 0));

  // Tiles [clean0, clean1) of the list are seen whole by every row of the wave, [whole0, whole1) by some row of the workgroup.
  const int clean0 = a.window > 0 ? tl.count_to(before(pos1, a.window), BN) - t0 : 0, clean1 = tl.count_to(pos0 - BN + 1, BN) - t0;
  const int whole0 = tl.count_to(tl.lo - 1, BN) - t0, whole1 = tl.count_to(tl.hi - BN + 1, BN) - t0;

  const int my_row = min(wrow + (int)r32, rt.rows - 1), my_tok = my_row / a.G, pos = rt.base + my_tok;

  // Staging. Wave w loads rows kWaveRows w .. of a tile. Pages hold 16 tokens or more, so they share one; a group of 16 of which
  // no row of q sees any is replaced by the nearest with one that some does. Lane i holds the offset in k and v of the rows of
  // tile 64 m + i of the workgroup's.
  const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
  constexpr uint32_t kLanes = kWave / kRowsPerLoad;  // of a row
  const uint32_t group_row = (kWaveRows * wave) & 15, lane_row = lane / kLanes, row_bytes = 2u * (uint32_t)p.token_stride;
  const uint32_t lane_off = lane_row * row_bytes, piece_k = 16u * (lane % kLanes ^ swizzle_k<T>(lane_row)),
                 piece_v = 16u * (lane % kLanes ^ swizzle_v<T>(lane_row));
  uint32_t at_lo = 0, at_hi = 0;
  // (the lane once more where the loop seldom comes: not held in a register through it)
  auto lane_again = [&]() __attribute__((always_inline)) {
    uint32_t x = lane_id();
    asm volatile("" : "+v"(x));
    return x;
  };
  auto look_up = [&](int first) __attribute__((always_inline)) {
    int g0 = (tl.start(t0 + min(first + (int)lane_again(), n - 1), BN) + kWaveRows * wave) & ~15;
    if (g0 >= tl.sinks) g0 = min(max(g0, tl.lo & ~15), tl.hi & ~15);
    int page = p.table[(int64_t)rt.b * p.max_pages + (g0 >> p.log2_page)];
    if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
    const int64_t at = 2 * ((int64_t)page * p.page_stride + (int64_t)h * p.head_stride +
                            (int64_t)((g0 & ((1 << p.log2_page) - 1)) + (int)group_row) * p.token_stride);
    at_lo = (uint32_t)at;
    at_hi = (uint32_t)(at >> 32);
  };
  auto stage_load = [&](const void* base, uint32_t piece, bool values, int buf, int i) __attribute__((always_inline)) {
    // (the places' XORs are linear in the row's bits: this load's share of them)
    const uint32_t r = kWaveRows * wave + kRowsPerLoad * i, x = 16u * (values ? swizzle_v<T>(r) : swizzle_k<T>(r));
    load_to_lds(base, lane_off + kRowsPerLoad * i * row_bytes + (piece ^ x),
                lds0 + (uint32_t)(buf + (values ? kRing : 0)) * kBuf + (kWaveRows * wave + kRowsPerLoad * i) * kRow);
  };
  // Where the keys of tile t (behind the last: the last, for nothing) lie; the values of the tile before lay where its keys did.
  uint64_t k_at = 0, v_at = 0;
  auto place = [&](int t) __attribute__((always_inline)) {
    t = min(t, n - 1);
    if (t % kWave == 0) look_up(t);
    v_at = k_at;
    k_at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at_hi, t % kWave) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)at_lo, t % kWave);
  };
  int k_buf = 0, v_buf = 0;  // where the next keys and values go
  // Load i of the 2 kLoads of a pair.
  auto stage = [&](int i) __attribute__((always_inline)) {
    uint32_t piece = i < kLoads ? piece_k : piece_v;
    asm volatile("" : "+v"(piece));  // (kept in registers for every load, the addresses would fill them)
    if (i < kLoads) stage_load(reinterpret_cast<const unsigned char*>(p.k) + k_at, piece, false, k_buf, i);
    else stage_load(reinterpret_cast<const unsigned char*>(p.v) + v_at, piece, true, v_buf, i - kLoads);
  };
  int placed = 0;  // the pair whose loads are next
  auto next_pair = [&]() __attribute__((always_inline)) {
    ++placed;
    place(placed + 1);
    k_buf = k_buf + 1 == kRing ? 0 : k_buf + 1;
    v_buf = v_buf + 1 == kRing ? 0 : v_buf + 1;
  };
  auto stage_pair = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2 * kLoads; ++i) stage(i);
    next_pair();
  };
  // This wave's rows of the values of tile t, which have arrived: what no row of q sees is cleared (it may be what memory held: 0
  // times that is not 0).
  auto clear_values = [&](int t) __attribute__((always_inline)) {
    if (t >= n || (t >= whole0 && t < whole1)) return;
    const int j0 = tl.start(t0 + t, BN);
    const uint32_t lane = lane_again(), lane_row = lane / kLanes;
    uint32_t zero_at = lds0 + (uint32_t)(kRing + t % kRing) * kBuf + kWaveRows * wave * kRow + 16 * lane;
#pragma unroll 1
    for (int i = 0; i < kLoads; ++i, zero_at += kRowsPerLoad * kRow) {
      const int x = j0 + kWaveRows * wave + kRowsPerLoad * i + (int)lane_row;
      if (x > tl.hi || (x < tl.lo && x >= tl.sinks))
        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(zero_at) = (u32x4){0u, 0u, 0u, 0u};
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  // Opens a step: the pair of the one behind it has arrived for every wave.
  int slot = 0;
  auto arrive = [&]() __attribute__((always_inline)) {
    wait_loads<2 * kLoads * (kDepth - 2)>();
    ++slot;
    clear_values(slot);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  const float inv_scale = 1.f / a.scale_log2;
  float l = 0.f, shift = 0.f, limit = -INFINITY;
  f32x16 o[ND];
#pragma unroll
  for (int c = 0; c < ND; ++c) o[c] = (f32x16){};

  // Operand i of the scores (tokens 32 (i % NK) .., channels 16 (i / NK) ..) and of the outputs (channels 32 (i % ND) .., tokens
  // 16 (i / ND) .., k slot 8 half + i being token 8 (i / 4) + 4 half + i % 4, as the scores lie). A row of LDS is a
  // multiple of its pieces' places, so that XOR selects the piece. (kAhead products: 2 and 6 are no faster, and from 4 on
  // registers spill at d = 128.)
  constexpr int kS = NK * NC, kO = 2 * NK * ND, kAhead = 3;
  const uint32_t kaddr = lds0 + r32 * kRow + 16u * (half ^ swizzle_k<T>(r32));
  const uint32_t vrow = 4 * half + (lane % 16) / 4;
  const uint32_t vaddr = lds0 + kRing * kBuf + vrow * kRow + 16u * ((((lane / 16) & 1) * 2 + (lane % 4) / 2) ^ swizzle_v<T>(vrow)) + 8 * (lane & 1);
  auto load_k = [&](uint32_t at, int i) __attribute__((always_inline)) { return lds_load<u32x4>((at ^ (32u * (i / NK))) + 32 * (i % NK) * kRow); };
  auto load_v = [&](uint32_t at, int i) __attribute__((always_inline)) {
    const uint32_t x = (at ^ (64u * (i % ND))) + 16 * (i / ND) * kRow;
    const u32x2 lo = lds_load_tr(x), hi = lds_load_tr(x + 8 * kRow);
    return (u32x4){lo.x, lo.y, hi.x, hi.y};
  };

  // The scores of tile t are masked and the shift follows them: limit is the largest score that it leaves alone (-inf before the
  // first), a row's other lane has the same.
  auto settle = [&](int t, f32x16 (&s)[NK]) __attribute__((always_inline)) {
    if (t < clean0 || t >= clean1) {
      const uint32_t half = lane_again() / 32;
      const int j0 = tl.start(t0 + t, BN), back = pos - j0 - 4 * (int)half;  // of this lane's first token of the tile
      if (a.window == 0) {
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[n][r] = back < 32 * n + 8 * (r / 4) + r % 4 ? -INFINITY : s[n][r];
      } else {
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int j = j0 + 32 * n + 8 * (r / 4) + 4 * (int)half + r % 4;
            if (!sees(pos, j, a.window, a.sinks)) s[n][r] = -INFINITY;
          }
      }
    }
    float top = max_of<NK>(s);
    if (ballot(top > limit)) {
      top = max_halves(top);
      const bool move = top > limit;
      const float to = move ? fmaf(-top, a.scale_log2, kBias) : shift;
      const float alpha = limit > -INFINITY ? __builtin_amdgcn_exp2f(to - shift) : 1.f;  // (nothing is there before the start)
      if (move) limit = fmaf(kSlack, inv_scale, top);
      shift = to;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < ND; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][r] *= alpha;
    }
  };
  // A tile's probabilities (in place of the scores), rounded one pair behind: the sum is that of the rounded ones. One rounding to
  // the type, whose errors are each weight's own, at most half a step of it, and make an output's 1.25 to 1.4 times its own
  // rounding's. In two parts, as k_paged_rows has them, the products with the values are twice as many: 4 prompts of 4096
  // tokens with 32 heads took 748 us for 551, 512 tokens behind 16384 203 for 153, 13 registers spilled.
  u32x4 pb[2 * NK];
  auto weights = [&](f32x16 (&s)[NK]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i <= 8 * NK; ++i) {
      if (i < 8 * NK)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          s[i / 8][2 * (i % 8) + e] = __builtin_amdgcn_exp2f(fmaf(s[i / 8][2 * (i % 8) + e], a.scale_log2, shift));
        }
      if (i == 0) continue;
      const int k = i - 1;
      const uint32_t xy = pack2<BF16>(s[k / 8][2 * (k % 8)], s[k / 8][2 * (k % 8) + 1]);
      l = add_pair<BF16>(xy, l);
      pb[k / 4][k % 4] = xy;
    }
  };
  u32x4 qb[NC];  // Q as the B operand: column = row of the wave, k = 16 c + 8 half + i
  u32x4 kf[kAhead], vf[kAhead];
  int kr = 1, vr = 0;  // the buffers of tile t + 1's keys and tile t's values
  // Step t with a tile behind it. Operands are read kAhead products before they are used (the first of X in the Y before).
  auto step = [&](int t, f32x16 (&s)[NK], f32x16 (&sn)[NK]) __attribute__((always_inline)) {
    arrive();
    uint32_t kat = kaddr + (uint32_t)kr * kBuf, vat = vaddr + (uint32_t)vr * kBuf;
    asm volatile("" : "+v"(kat), "+v"(vat));  // (as in stage)
#pragma unroll
    for (int i = 0; i < kS; ++i) {
      sn[i % NK] = mfma32<BF16>(kf[i % kAhead], qb[i / NK], i < NK ? (f32x16){} : sn[i % NK]);
      if (i < 2 * kLoads) stage(i);
      if (i + kAhead < kS) kf[i % kAhead] = load_k(kat, i + kAhead);
      else vf[i + kAhead - kS] = load_v(vat, i + kAhead - kS);
      __builtin_amdgcn_sched_barrier(0);
    }
    next_pair();
    weights(s);
    kr = kr + 1 == kRing ? 0 : kr + 1;
    vr = vr + 1 == kRing ? 0 : vr + 1;
    uint32_t knext = kaddr + (uint32_t)kr * kBuf;
    asm volatile("" : "+v"(vat), "+v"(knext));
#pragma unroll
    for (int i = 0; i < kO; ++i) {
      o[i % ND] = mfma32<BF16>(vf[i % kAhead], pb[i / ND], o[i % ND]);
      if (i + kAhead < kO) vf[i % kAhead] = load_v(vat, i + kAhead);
      else kf[i + kAhead - kO] = load_k(knext, i + kAhead - kO);
      __builtin_amdgcn_sched_barrier(0);
    }
    settle(t + 1, sn);
  };
  // The wave's last step.
  auto finish = [&](f32x16 (&s)[NK]) __attribute__((always_inline)) {
    arrive();
    stage_pair();
    __builtin_amdgcn_sched_barrier(0);
    uint32_t vat = vaddr + (uint32_t)vr * kBuf;
    asm volatile("" : "+v"(vat));
#pragma unroll
    for (int i = 0; i < kAhead; ++i) vf[i] = load_v(vat, i);
    weights(s);
#pragma unroll
    for (int i = 0; i < kO; ++i) {
      o[i % ND] = mfma32<BF16>(vf[i % kAhead], pb[i / ND], o[i % ND]);
      if (i + kAhead < kO) vf[i % kAhead] = load_v(vat, i + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (n > 0) {
    f32x16 s0[NK], s1[NK];
    // Where the tiles lie; q; the first tile's keys, then pairs 0 .. kDepth - 1: all under way at once.
    place(0);
    __builtin_amdgcn_sched_barrier(0);
    {
      const uint16_t* q = a.q + (int64_t)(rt.tok0 + my_tok) * a.q_stride + (h * a.G + my_row - my_tok * a.G) * d + 8 * half;
#pragma unroll
      for (int c = 0; c < NC; ++c) qb[c] = *reinterpret_cast<const u32x4*>(q + 16 * c);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) stage(i);
    k_buf = 1;
    place(1);
#pragma unroll 1
    for (int i = 0; i < kDepth; ++i) stage_pair();
    // (q's wait is here: inside the loop it would be one for the tiles' loads too)
    wait_loads<0>();
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(qb[c]));
    clear_values(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (mine > 0) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = load_k(kaddr, i);
#pragma unroll
      for (int i = 0; i < kS; ++i) {
        s0[i % NK] = mfma32<BF16>(kf[i % kAhead], qb[i / NK], i < NK ? (f32x16){} : s0[i % NK]);
        if (i + kAhead < kS) kf[i % kAhead] = load_k(kaddr, i + kAhead);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = load_k(kaddr + kBuf, i);
      settle(0, s0);
      int t = 0;
      for (; t + 2 < mine; t += 2) {
        step(t, s0, s1);
        step(t + 1, s1, s0);
      }
      if (t + 1 < mine) {
        step(t, s0, s1);
        finish(s1);
      } else {
        finish(s0);
      }
    }
    // Steps of the other waves; none may end while its loads are under way.
    while (slot < n) {
      arrive();
      stage_pair();
    }
    wait_loads<0>();
  }

  const uint32_t lane2 = lane_again();
  const int row = wrow + (int)(lane2 % 32), half4 = 4 * (int)(lane2 / 32);
  l += __shfl_xor(l, 32, kWave);
  float z = l * 0.f;  // NaN if something is not finite
#pragma unroll
  for (int c = 0; c < ND; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = fmaf(o[c][r], 0.f, z);
  if (ballot(row < rt.rows && (z != z || fabsf(shift) >= kFar<BF16>))) {
    redo_rows<T, BF16>(a, part, rt, h, wrow, 32, tl, t0, t0 + n, split, BN);
    return;
  }
  const int tok = row / a.G, hq = h * a.G + (row - tok * a.G);
  const int64_t t = rt.tok0 + tok;
  const bool nothing = rt.base + tok < 0;
  if (part.n_splits > 1) {
    if (row >= rt.rows) return;
    const int64_t orow = (int64_t)split * a.n_q * a.Hq + t * a.Hq + hq;
    if (half4 == 0) part.ml[orow] = make_float2(limit > -INFINITY ? -shift : -INFINITY, nothing ? -1.f : l);
    float* dst = part.o + orow * d + half4;
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<f32x4*>(dst + 32 * c + 2 * r) = (f32x4){o[c][r], o[c][r + 1], o[c][r + 2], o[c][r + 3]};
  } else {
    // Eight channels a lane: its own four and the row's other lane's, of each 16.
    const float inv = nothing ? 0.f : 1.f / l;
    uint16_t* dst = a.out + t * a.out_stride + hq * d + 2 * half4;
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 8) {
        uint32_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = pack2<BF16>(o[c][r + 2 * e] * inv, o[c][r + 2 * e + 1] * inv);
        const auto lo = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
        if (row < rt.rows)
          *reinterpret_cast<u32x4*>(dst + 32 * c + 2 * r) = (u32x4){(uint32_t)lo[0], (uint32_t)hi[0], (uint32_t)lo[1], (uint32_t)hi[1]};
      }
  }
}

// ------------------------------------------------------------------------------------------
// k_paged_rows: at most 16 rows, one wave, tiles of 32 tokens: single tokens (and few) over a long cache.
//
// The loads bound it (16 KB of keys and values a tile at d = 128 for some 180 vector instructions), so nothing goes through
// LDS: a key row's 16-byte pieces are the A operand of S = K Q^T as they are loaded (lane = token l % 16, channels 32 c +
// 8 (l / 16)), its result (row l % 16, tokens 4 (l / 16) + e of the tile's two groups of 16) is the A operand of O = P V, and a
// lane loads channels 4 T (l % 16) .. of those eight tokens and transposes them with byte permutes into the B operand.
//
// The loads leave the matrix units room for the probabilities in two parts of the type, so that 16 bits of them are left in bf16 and
// 22 in fp16, and the sum is that of the unrounded ones: 18.4 us for 18.2, 118.3 for 117.7 and 21.2 for 21.0 on the first three
// calls below, both forms in turn on one card. Rounded to the type they made bf16 outputs' error 1.4 times their own rounding's.
//
// With k_paged_merge, and in parentheses k_paged_chunk instead: 16 requests of up to 16384 tokens, 8 kv-heads of 4 rows, d = 128 (634
// MB) 116 us, 5.5 TB/s (152); one of 4096 with 32 heads 18.4 (20.5); 32 with a window of 1024, d = 64, 8 rows 21.5 (21); of 16
// rows, 16 requests of 16384 tokens 166 (194), one 23.6 (22), 32 of 1024 32.6 (28). Rows beyond 16 would read the pages twice. The next
// tile's loads follow the products that free their registers; with as many registers again, for two tiles: 119 us for 117.
// ------------------------------------------------------------------------------------------
constexpr int kRowsTile = 32;

template <bool BF16>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

template <int T, bool BF16>
__global__ __launch_bounds__(kWave) void k_paged_rows(PagedAttnArgs a, PartOut part) {
  constexpr int d = kTile * T, NC = 2 * T, NO = 4 * T, BN = kRowsTile;
  const PagedView& p = a.p;
  const int h = blockIdx.x % p.H, split = (blockIdx.x / p.H) % part.n_splits, tile = blockIdx.x / (p.H * part.n_splits);
  const RowTile rt = a.mixed ? rows_of(a, tile) : row_tile<kFewRows>(a, tile, false);
  if (rt.row0 >= rt.rows || (a.mixed && rt.rows > kFewRows)) return;
  const uint32_t lane = lane_id(), r16 = lane % 16, q4 = lane / 16;
  const int row = min(rt.row0 + (int)r16, rt.rows - 1), tok = row / a.G, pos = rt.base + tok;
  const int pos0 = rt.base + rt.row0 / a.G, pos1 = rt.base + (min(rt.row0 + kFewRows, rt.rows) - 1) / a.G;
  const TileList tl(pos0, pos1, a.window, a.sinks, BN);
  const int t0 = (int)((int64_t)tl.n * split / part.n_splits);
  const int n = (int)((int64_t)tl.n * (split + 1) / part.n_splits) - t0;
  // Tiles [clean0, clean1) are seen whole by every row, [whole0, whole1) by some.
  const int clean0 = a.window > 0 ? tl.count_to(before(pos1, a.window), BN) - t0 : 0, clean1 = tl.count_to(pos0 - BN + 1, BN) - t0;
  const int whole0 = tl.count_to(tl.lo - 1, BN) - t0, whole1 = tl.count_to(tl.hi - BN + 1, BN) - t0;

  // Lane i holds the offset in k and v of group i of 16 tokens of the 32 tiles at hand (one that no row sees is replaced by the
  // nearest that some row does; pages hold 16 tokens or more).
  uint32_t at_lo = 0, at_hi = 0;
  const uint32_t row_bytes = 2u * (uint32_t)p.token_stride;
  auto group_of = [&](int t, int g) __attribute__((always_inline)) {
    const int g0 = tl.start(t0 + t, BN) + 16 * g;
    return g0 < tl.sinks ? g0 : min(max(g0, tl.lo & ~15), tl.hi & ~15);
  };
  auto look_up = [&](int first) __attribute__((always_inline)) {
    const int g0 = group_of(min(first + (int)lane / 2, n - 1), lane & 1);
    int page = p.table[(int64_t)rt.b * p.max_pages + (g0 >> p.log2_page)];
    if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
    const int64_t at = 2 * ((int64_t)page * p.page_stride + (int64_t)h * p.head_stride +
                            (int64_t)(g0 & ((1 << p.log2_page) - 1)) * p.token_stride);
    at_lo = (uint32_t)at;
    at_hi = (uint32_t)(at >> 32);
  };
  auto base_of = [&](const uint16_t* x, int t, int g) __attribute__((always_inline)) {
    const int i = (2 * t + g) % kWave;
    return reinterpret_cast<const unsigned char*>(x) + ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at_hi, i) << 32 |
                                                        (uint32_t)__builtin_amdgcn_readlane((int)at_lo, i));
  };
  // Row r of a group of a tile at the ends of what is seen: the nearest that some row sees (the others may be what memory held,
  // and 0 times that is not 0).
  auto nearest = [&](int r, int t, int g) __attribute__((always_inline)) {
    const int g0 = group_of(t, g);
    const bool first = g0 < tl.sinks;
    const int from = first ? 0 : tl.lo, to = first && tl.lo > g0 + 15 ? tl.sinks - 1 : tl.hi;
    return min(max(r, from - g0), min(to - g0, 15));
  };
  u32x4 kr[2][NC];
  uint32_t vr[8][2 * T];
  auto load_keys = [&](int t) __attribute__((always_inline)) {
    if (t % (kWave / 2) == 0) look_up(t);
    const bool edge = t < whole0 || t >= whole1;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t r = r16;
      if (edge) r = (uint32_t)nearest((int)r, t, g);
      const unsigned char* x = base_of(p.k, t, g) + (r * row_bytes + 16u * q4);
#pragma unroll
      for (int c = 0; c < NC; ++c) kr[g][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x + 64 * c));
    }
  };
  auto load_values = [&](int t) __attribute__((always_inline)) {
    const bool edge = t < whole0 || t >= whole1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t r = 4 * q4 + i % 4;
      if (edge) r = (uint32_t)nearest((int)r, t, i / 4);
      const unsigned char* x = base_of(p.v, t, i / 4) + (r * row_bytes + 2u * NO * r16);
      if constexpr (T == 1) {
        const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(x));
        vr[i][0] = v.x;
        vr[i][1] = v.y;
      } else {
#pragma unroll
        for (int m = 0; m < T / 2; ++m) {
          const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x) + m);
          vr[i][4 * m] = v.x;
          vr[i][4 * m + 1] = v.y;
          vr[i][4 * m + 2] = v.z;
          vr[i][4 * m + 3] = v.w;
        }
      }
    }
  };

  const float inv_scale = 1.f / a.scale_log2;
  float l = 0.f, shift = 0.f, limit = -INFINITY;
  f32x4 o[NO];
#pragma unroll
  for (int c = 0; c < NO; ++c) o[c] = (f32x4){};
  if (n > 0) {
    load_keys(0);
    u32x4 qb[NC];  // Q as the B operand: column = row, k = 32 c + 8 (l / 16) + i
    {
      const uint16_t* q = a.q + (int64_t)(rt.tok0 + tok) * a.q_stride + (h * a.G + row - tok * a.G) * d + 8 * q4;
#pragma unroll
      for (int c = 0; c < NC; ++c) qb[c] = *reinterpret_cast<const u32x4*>(q + 32 * c);
    }
    load_values(0);
    for (int t = 0; t < n; ++t) {
      f32x4 s[2] = {};
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int c = 0; c < NC; ++c) s[g] = mfma16<BF16>(kr[g][c], qb[c], s[g]);
      // (the values of the tile whose offsets this may replace are loaded already)
      if (t + 1 < n) load_keys(t + 1);
      if (t < clean0 || t >= clean1) {
        const int j0 = tl.start(t0 + t, BN) + 4 * (int)q4;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!sees(pos, j0 + 16 * g + e, a.window, a.sinks)) s[g][e] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e / 4][e % 4]);
      if (ballot(top > limit)) {
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const bool move = top > limit;
        const float to = move ? fmaf(-top, a.scale_log2, kBias) : shift;
        const float alpha = limit > -INFINITY ? __builtin_amdgcn_exp2f(to - shift) : 1.f;
        if (move) limit = fmaf(kSlack, inv_scale, top);
        shift = to;
        l *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float ae = __shfl(alpha, (int)(4 * q4) + e, kWave);  // row 4 (l / 16) + e of the outputs
#pragma unroll
          for (int c = 0; c < NO; ++c) o[c][e] *= ae;
        }
      }
      u32x4 pa, pl;  // the probabilities in two parts of the type, the second what the first leaves
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[e / 2][2 * (e % 2)], a.scale_log2, shift));
        const float y = __builtin_amdgcn_exp2f(fmaf(s[e / 2][2 * (e % 2) + 1], a.scale_log2, shift));
        pa[e] = pack2<BF16>(x, y);
        pl[e] = pack2<BF16>(x - to_float<BF16>(pa[e] & 0xffffu), y - to_float<BF16>(pa[e] >> 16));
        l += x + y;
      }
#pragma unroll
      for (int c = 0; c < NO; ++c) {
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = __builtin_amdgcn_perm(vr[2 * i + 1][c / 2], vr[2 * i][c / 2], (c & 1) ? 0x07060302u : 0x05040100u);
        const u32x4 v = {y[0], y[1], y[2], y[3]};
        o[c] = mfma16<BF16>(pl, v, mfma16<BF16>(pa, v, o[c]));
      }
      if (t + 1 < n) load_values(t + 1);
    }
  }

  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  float z = l * 0.f;  // NaN if something is not finite
#pragma unroll
  for (int c = 0; c < NO; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (rt.row0 + (int)(4 * q4) + e < rt.rows) z = fmaf(o[c][e], 0.f, z);
  if (ballot(z != z || (rt.row0 + (int)r16 < rt.rows && fabsf(shift) >= kFar<BF16>))) {
    redo_rows<T, BF16>(a, part, rt, h, rt.row0, kFewRows, tl, t0, t0 + n, split, BN);
    return;
  }
  if (part.n_splits > 1 && q4 == 0 && rt.row0 + (int)r16 < rt.rows)
    part.ml[split * part.rows + part_row(a, part, rt, h, row)] =
        make_float2(limit > -INFINITY ? -shift : -INFINITY, pos < 0 ? -1.f : l);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int orow = rt.row0 + (int)(4 * q4) + e, otok = orow / a.G, hq = h * a.G + orow - otok * a.G;
    const float le = __shfl(l, (int)(4 * q4) + e, kWave);
    if (orow >= rt.rows) continue;
    const int64_t t = rt.tok0 + otok;
    if (part.n_splits > 1) {
      f32x4* dst = reinterpret_cast<f32x4*>(part.o + (split * part.rows + part_row(a, part, rt, h, orow)) * d + NO * r16);
#pragma unroll
      for (int c = 0; c < T; ++c) dst[c] = (f32x4){o[4 * c][e], o[4 * c + 1][e], o[4 * c + 2][e], o[4 * c + 3][e]};
    } else {
      const float inv = rt.base + otok < 0 ? 0.f : 1.f / le;
      u32x2* dst = reinterpret_cast<u32x2*>(a.out + t * a.out_stride + hq * d + NO * r16);
#pragma unroll
      for (int c = 0; c < T; ++c)
        dst[c] = (u32x2){pack2<BF16>(o[4 * c][e] * inv, o[4 * c + 1][e] * inv), pack2<BF16>(o[4 * c + 2][e] * inv, o[4 * c + 3][e] * inv)};
    }
  }
}

// ------------------------------------------------------------------------------------------
// k_paged_merge: the ranges of a row together, out = sum w o / sum w l with w = 2^(m - max m).
//
// A stream of d / 4 lanes loads a range's outputs, four a lane, kMergeAhead ranges at once and the first ones before the weights
// are known; OF lanes look at the weights. A row has one stream, or, where rows are few and ranges many (WIDE), the 16 / T of a
// workgroup, each with every (16 / T)-th range, which shuffles and LDS add up. Latency bounds it: 4 us for up to 500 rows; at
// d = 128, 16384 rows of 4 ranges take 9.4 us (3.8 TB/s; 12.5 with a wave a row). One stream a row against a workgroup a row:
// 32 rows of 256 ranges 23.4 and 7.2 us, 512 of 16 4.8 both, 992 of 8 to 16 6.5 and 7.8, 2404 of 21 7.6 and 13.0.
// ------------------------------------------------------------------------------------------
constexpr int kMergeAhead = 8, kMergeWideRows = 512;

template <int T, bool BF16, int OF, bool WIDE>
__global__ __launch_bounds__(kMergeThreads) void k_paged_merge(PagedAttnArgs a, PartOut part, int of_few) {
  constexpr int d = kTile * T, L = 16 * T, S = kMergeThreads / L;
  constexpr int kStep = WIDE ? S : 1, kAhead = kMergeAhead < OF / kStep ? kMergeAhead : OF / kStep;
  static_assert(OF % (kStep * kAhead) == 0, "the ranges under way are of one round of weights");
  const int lane = (int)lane_id(), stream = (int)threadIdx.x / L, sub = (int)threadIdx.x % L;
  const int64_t rows = part.rows, i0 = WIDE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * S + stream;
  // The row: of q and all its heads, or, where the requests of few rows have ranges of their own, the r-th of a request's and kv-head's.
  int t, hq;
  bool mine;
  if (a.mixed && of_few) {
    const int r = (int)(i0 % kFewRows), h = (int)(i0 / kFewRows % a.p.H), b = (int)(i0 / kFewRows / a.p.H);
    if (b >= a.p.B) return;
    const RowTile rt = rows_of(a, b);  // (a wave's rows are one request's: S divides kFewRows)
    mine = r < rt.rows && rt.rows <= kFewRows;
    t = rt.tok0 + r / a.G;
    hq = h * a.G + r % a.G;
  } else {
    t = (int)(i0 / a.Hq);
    hq = (int)(i0 - (int64_t)t * a.Hq);
    mine = i0 < (int64_t)a.n_q * a.Hq && t < a.cu[a.p.B];
    if (a.mixed) {
#pragma unroll
      for (int k = 0; k < (WIDE ? 1 : kWave / L); ++k) {
        const int x = __builtin_amdgcn_readlane(t, k * L);
        const bool few = request_of(a, x).rows <= kFewRows;
        if (x == t && few) mine = false;
      }
    }
  }
  if (!mine) return;  // (all of a stream; WIDE: all of the workgroup)
  const int64_t row = part.by_entry ? i0 : (int64_t)t * a.Hq + hq;
  const int first = WIDE ? stream : 0, at = lane % OF;
  f32x4 x[kAhead], o = {};
  auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (s0 + kStep * k < part.n_splits) x[k] = *reinterpret_cast<const f32x4*>(part.o + ((s0 + kStep * k) * rows + row) * d + 4 * sub);
  };
  load(first);
  float M = -INFINITY, l = 0.f;
  for (int s = at; s < part.n_splits; s += OF) M = fmaxf(M, part.ml[s * rows + row].x);
#pragma unroll
  for (int k = 1; k < OF; k *= 2) M = fmaxf(M, __shfl_xor(M, k, kWave));
  uint64_t nothing = 0;
  for (int s0 = 0; s0 < part.n_splits; s0 += OF) {
    // lane i of those: the weight of range s0 + i, 0 for one without any (its output is not looked at)
    float2 ml = make_float2(-INFINITY, 0.f);
    if (s0 + at < part.n_splits) ml = part.ml[(s0 + at) * rows + row];
    const float w = ml.x != -INFINITY || ml.y != 0.f ? at_least(__builtin_amdgcn_exp2f(ml.x - M)) : 0.f;
    if (w != 0.f) l = fmaf(ml.y, w, l);
    nothing |= ballot(ml.y < 0.f);
    const int end = min(s0 + OF, part.n_splits);
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

template <int T, bool BF16>
static hipError_t merge_launch(const PagedAttnArgs& a, const PartOut& part, bool of_few, hipStream_t s) {
  if (part.n_splits <= 1) return hipSuccess;  // (written by its kernel)
  const int64_t rows = a.mixed && of_few ? (int64_t)a.p.B * a.p.H * kFewRows : (int64_t)a.n_q * a.Hq;
  const dim3 streams((uint32_t)merge_groups(rows, T)), block(kMergeThreads);
  if (part.n_splits <= kMergeAhead)
    hipLaunchKernelGGL((k_paged_merge<T, BF16, kMergeAhead, false>), streams, block, 0, s, a, part, (int)of_few);
  else if (rows >= kMergeWideRows)
    hipLaunchKernelGGL((k_paged_merge<T, BF16, 16 * T, false>), streams, block, 0, s, a, part, (int)of_few);
  else
    hipLaunchKernelGGL((k_paged_merge<T, BF16, kWave, true>), dim3((uint32_t)rows), block, 0, s, a, part, (int)of_few);
  return hipGetLastError();
}

template <int T, bool BF16>
static hipError_t attn_launch(const PagedAttnArgs& a, hipStream_t s) {
  // (all outputs first, aligned as they are accessed)
  const int64_t rows = (int64_t)a.n_q * a.Hq, n_few = paged_parts(a.few_rows, a.few), n_many = paged_parts(rows, a.many);
  float* const o = (float*)a.ws;
  float2* const ml = (float2*)(o + (n_few + n_many) * (64 * T));
  const PartOut few = {ml, o, a.few_rows, a.by_entry, a.few}, many = {ml + n_few, o + n_few * (64 * T), rows, 0, a.many};
  hipError_t e;
  if (a.few > 0) {
    const int64_t tiles = a.mixed ? a.p.B : paged_tiles(a.p, a.G, a.n_q, kFewRows);
    hipLaunchKernelGGL((k_paged_rows<T, BF16>), dim3((uint32_t)(tiles * a.p.H * a.few)), dim3(kWave), 0, s, a, few);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.many > 0) {
    const int64_t tiles = paged_tiles(a.p, a.G, a.n_q, chunk_rows(T));
    hipLaunchKernelGGL((k_paged_chunk<T, BF16>), dim3((uint32_t)(tiles * a.p.H * a.many)), dim3(kWave * chunk_waves(T)), 0, s,
                       a, many);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if ((e = merge_launch<T, BF16>(a, few, true, s)) != hipSuccess) return e;
  return merge_launch<T, BF16>(a, many, false, s);
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.p.d) {
    case 64: return a.p.bf16 ? attn_launch<1, true>(a, s) : attn_launch<1, false>(a, s);
    case 128: return a.p.bf16 ? attn_launch<2, true>(a, s) : attn_launch<2, false>(a, s);
    default: return a.p.bf16 ? attn_launch<4, true>(a, s) : attn_launch<4, false>(a, s);
  }
}

}  // namespace mf
