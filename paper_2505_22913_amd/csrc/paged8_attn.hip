// Causal attention of the new tokens of every request over its pages of 8-bit codes (gfx950), with an
// optional sliding window and first tokens that stay visible.
#include "codes.h"
#include "paged8.h"

namespace mf {

// A token's key and value for one_row().
template <bool INT8>
struct Pages8 {
  struct Held {
    int64_t at;
    float ks, vs;
  };
  const Paged8AttnArgs& a;
  __device__ __forceinline__ Held held(int page, int h, int place) const {
    const PagedView& p = a.p;
    const int64_t block = (((int64_t)page * p.H + h) << (p.log2_page - a.log2_block)) + (place >> a.log2_block);
    return {(int64_t)page * p.page_stride + (int64_t)h * p.head_stride + (int64_t)place * p.token_stride, power_of(a.k_scale[block]),
            power_of(a.v_scale[block])};
  }
  __device__ __forceinline__ float code(const uint16_t* x, int64_t i) const {
    return decode4<INT8>(reinterpret_cast<const uint8_t*>(x)[i], 1.f)[0];
  }
  __device__ __forceinline__ float key(const Held& t, int c) const { return code(a.p.k, t.at + c) * t.ks; }
  __device__ __forceinline__ Held passed(const Held& t, int lane) const {
    return {(int64_t)__shfl(t.at, lane, kWave), 0.f, __shfl(t.vs, lane, kWave)};
  }
  __device__ __forceinline__ float value(const Held& t, int c) const { return code(a.p.v, t.at + c) * t.vs; }
};

// Tile `tile` of the launch, of which not every one is one: n rows are in n / BM + 1 tiles at most, so that a request's may begin at its
// first row / BM + b, and the next one's behind them. To count the requests' tiles, so that those without work come last, takes
// each workgroup two loads after each other for every 64 of them: chunks of 20 tokens of every second request and single tokens of the
// others, 65 of them 44 us for 57, 500 168 for 153, 4096 with 8 kv-heads 2.6 ms for 0.84; single tokens alone, 4096, 118 us for 38.
constexpr int kCounted = 256;
template <int BM>
__device__ __forceinline__ RowTile spread_tile(const PagedAttnArgs& a, int tile) {
  auto start = [&](int cu, int b) { return (int)((int64_t)cu * a.G / BM) + b; };
  const Request r = last_request(a.cu, a.p.state, a.p.B, [&](int cu, int b) { return start(cu, b) <= tile; });
  RowTile rt = rows_at(a, r.b, r.cu, r.next, r.len);
  rt.row0 = tile < start(r.cu, r.b) ? rt.rows : (tile - start(r.cu, r.b)) * BM;
  return rt;
}

// Tile s n / of of n tiles in `of` ranges (at most 2^16), in 32 bits.
__device__ __forceinline__ int range_start(int n, int s, int of) {
  return n / of * s + (int)((uint32_t)(n % of) * (uint32_t)s / (uint32_t)of);
}

// ------------------------------------------------------------------------------------------
// k_paged8_chunk: 32 rows a wave, 8 waves a workgroup (4 at d = 256), tiles of 64 tokens (32): chunks of prompts.
//
// The products are k_paged_chunk's, over tiles of values in LDS. Codes become values once a workgroup: a tile's codes arrive in LDS
// by direct loads, three steps ahead, each wave converts the rows that it has loaded itself (so their arrival needs no
// barrier) and stores them where the products read them; the step's one barrier hands them to the others. Pair p is the codes
// of the keys of tile p + 3 and of the values of tile p + 1; step t converts pair t, a piece at a time between the products, and
// loads pair t + 3 in its place. So three buffers of keys do (one that X reads, the next one, whose first operands are read before
// the barrier, and the one that is written) and two of values.
//
// 4 d flops a visible pair bound it, and the matrix and vector units hardly work at once: 4 prompts of 4096 tokens with 32 heads of 128
// (550 GFLOP, e4m3, bf16) 566 to 604 us, 0.91 to 0.97 PFLOP/s, where a product of 8192^3 reaches 1.25; 512 rows of 4 heads a kv-head
// behind 16384 tokens (int8, fp16) 151 to 165 with their join. The same from 16-bit pages: 548 to 568 and 148 to 155; the difference
// is the conversion, 27% more vector instructions, and its stores to LDS (a sixth of LDS's cycles are their conflicts). With 16
// rows a wave that converts its operands for itself they took 1766 us and 897. The probabilities are rounded to the type once:
// errors against 64 bits 0.0021 for 0.0016 in bf16, 0.00029 for 0.00021 in fp16 (2-norms, relative); in two parts the products of the
// outputs would double.
// ------------------------------------------------------------------------------------------
constexpr int kKeyBufs = 3, kValueBufs = 2, kCodeBufs = 3;

template <int T, bool BF16, bool INT8>
__global__ __launch_bounds__(chunk_waves(T) * kWave, T == 4 ? 1 : 2) void k_paged8_chunk(Paged8AttnArgs a, PartOut part) {
  constexpr int NW = chunk_waves(T), BM = 32 * NW;
  constexpr int d = kTile * T, BN = chunk_tile<T>(), NK = BN / 32, NC = d / 16, ND = d / 32;
  constexpr uint32_t kRow = 2 * d, kBuf = BN * kRow, kCodes = BN * d;  // bytes
  constexpr int kWaveRows = BN / NW, kLanes = d / 16;                  // rows of a tile that a wave loads, lanes of a row
  constexpr int kRowsPerLoad = kWave / kLanes < kWaveRows ? kWave / kLanes : kWaveRows, kLoads = kWaveRows / kRowsPerLoad;
  constexpr int kActive = kRowsPerLoad * kLanes;  // lanes of a load
  static_assert(kLoads * kRowsPerLoad == kWaveRows && 16 % kWaveRows == 0, "a wave's rows");
  __shared__ __align__(1024) unsigned char smem[(kKeyBufs + kValueBufs) * kBuf + kCodeBufs * 2 * kCodes];
  const PagedView& p = a.p;
  const int h = blockIdx.x % p.H, split = (blockIdx.x / p.H) % part.n_splits, tile = (int)(blockIdx.x / (p.H * part.n_splits));
  const RowTile rt = a.p.B <= kCounted ? row_tile<BM>(a, tile, a.mixed != 0) : spread_tile<BM>(a, tile);
  if (rt.row0 >= rt.rows || (a.mixed && rt.rows <= kFewRows)) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const uint32_t lane = lane_id(), r32 = lane % 32, half = lane / 32;
  const int wrow = rt.row0 + 32 * wave;  // the wave's first row
  const TileList tl(rt.base + rt.row0 / a.G, rt.base + (min(rt.row0 + BM, rt.rows) - 1) / a.G, a.window, a.sinks, BN);
  const int t0 = range_start(tl.n, split, part.n_splits), n = range_start(tl.n, split + 1, part.n_splits) - t0;  // tiles of the workgroup
  // The wave's rows' positions, and its tiles: those behind its last position are the others'.
  const int pos0 = rt.base + min(wrow, rt.rows - 1) / a.G, pos1 = rt.base + min(wrow + 31, rt.rows - 1) / a.G;
  const int mine = wrow >= rt.rows || pos1 < 0 ? 0 : min(n, max(tl.count_to(pos1, BN) - t0, 0));

  // Tiles [clean0, clean1) of the list are seen whole by every row of the wave, [whole0, whole1) by some row of the workgroup.
  const int clean0 = a.window > 0 ? tl.count_to(before(pos1, a.window), BN) - t0 : 0, clean1 = tl.count_to(pos0 - BN + 1, BN) - t0;
  const int whole0 = tl.count_to(tl.lo - 1, BN) - t0, whole1 = tl.count_to(tl.hi - BN + 1, BN) - t0;

  const int my_row = min(wrow + (int)r32, rt.rows - 1), my_tok = my_row / a.G, pos = rt.base + my_tok;

  // Staging. Wave w has rows kWaveRows w .. of a tile. Pages and blocks hold 16 tokens or more, so they share one; a group of 16 of
  // which no row of q sees any is replaced by the nearest with one that some does. Lane i holds the offset in k and v of the rows of
  // tile 64 m + i of the workgroup's, and their scale bytes.
  const uint32_t lds0 = (uint32_t)(uintptr_t)smem, codes0 = lds0 + (kKeyBufs + kValueBufs) * kBuf;
  const uint32_t group_row = (kWaveRows * wave) & 15, row_bytes = (uint32_t)p.token_stride;
  const uint32_t lane_off = lane / kLanes * row_bytes + 16u * (lane % kLanes);
  uint32_t at_lo = 0, at_hi = 0, scales = 0;
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
    const int place = g0 & ((1 << p.log2_page) - 1);
    const int64_t at = (int64_t)page * p.page_stride + (int64_t)h * p.head_stride + (int64_t)(place + (int)group_row) * p.token_stride;
    const int64_t block = (((int64_t)page * p.H + h) << (p.log2_page - a.log2_block)) + (place >> a.log2_block);
    at_lo = (uint32_t)at;
    at_hi = (uint32_t)(at >> 32);
    scales = (uint32_t)a.k_scale[block] | (uint32_t)a.v_scale[block] << 8;
  };
  // The tiles that were placed last (behind the workgroup's last: that one, for nothing), newest first: where the newest three lie,
  // and eight scale bytes of keys and of values.
  uint64_t at[3] = {}, k_bytes = 0, v_bytes = 0;
  int placed = 0;
  auto place = [&]() __attribute__((always_inline)) {
    const int t = min(placed++, n - 1);
    if (t % kWave == 0) look_up(t);
    at[2] = at[1];
    at[1] = at[0];
    at[0] = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at_hi, t % kWave) << 32 |
            (uint32_t)__builtin_amdgcn_readlane((int)at_lo, t % kWave);
    const uint32_t sc = (uint32_t)__builtin_amdgcn_readlane((int)scales, t % kWave);
    k_bytes = k_bytes << 8 | (sc & 0xffu);
    v_bytes = v_bytes << 8 | (sc >> 8 & 0xffu);
  };
  auto scale_of = [&](uint64_t bytes, int back) __attribute__((always_inline)) { return power_of((uint32_t)(bytes >> (8 * back)) & 0xffu); };
  int code_buf = 0, key_buf = 0, value_buf = 1;  // where the next pair's codes lie and go, where its keys and values go
  // Load i of the 2 kLoads of a pair, whose tiles are placed.
  auto stage = [&](int i) __attribute__((always_inline)) {
    const bool values = i >= kLoads;
    const int k = values ? i - kLoads : i;
    uint32_t off = lane_off + kRowsPerLoad * k * row_bytes;
    asm volatile("" : "+v"(off));
    const unsigned char* base = reinterpret_cast<const unsigned char*>(values ? p.v : p.k) + (values ? at[2] : at[0]);
    const uint32_t dst = codes0 + (uint32_t)(2 * code_buf + values) * kCodes + kWaveRows * wave * d + 16 * kActive * k;
    if (kActive == kWave || lane < kActive) load_to_lds(base, off, dst);
  };
  // Codes of this wave's rows as values where the products read them: 16 bytes of a row (its 8-token, 8-channel pieces are stored at
  // their place XOR the row's). What no row of q sees of a tile's values is cleared (it may be what memory held: 0 times that is not 0).
  auto store_half = [&](uint32_t dst, uint32_t w0, uint32_t w1, float scale) __attribute__((always_inline)) {
    const u32x2 x = decode_pairs<BF16, INT8>(w0, scale), y = decode_pairs<BF16, INT8>(w1, scale);
    *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(dst) = (u32x4){x.x, x.y, y.x, y.y};
  };
  auto piece_at = [&](bool values, int k) __attribute__((always_inline)) {
    const uint32_t row = kWaveRows * wave + kRowsPerLoad * k + lane / kLanes;
    return row * kRow + 16u * ((2 * (lane % kLanes)) ^ (values ? swizzle_v<T>(row) : swizzle_k<T>(row)));
  };
  auto unseen = [&](int t, int k) __attribute__((always_inline)) {
    const int x = tl.start(t0 + t, BN) + kWaveRows * wave + kRowsPerLoad * k + (int)(lane_again() / kLanes);
    return x > tl.hi || (x < tl.lo && x >= tl.sinks);
  };
  // Chores of step t, a few between each two products: the wave's codes of pair t have arrived.
  u32x4 raw;
  uint32_t raw_at = 0;
  constexpr int kChores = 6 * kLoads + 2 * kLoads;
  auto chore = [&](int t, int i) __attribute__((always_inline)) {
    if (i < 6 * kLoads) {
      const bool values = i >= 3 * kLoads;
      const int k = i % (3 * kLoads) / 3, part_of = i % 3;
      const float scale = values ? scale_of(v_bytes, 4) : scale_of(k_bytes, 2);
      if (part_of == 0) {
        raw_at = codes0 + (uint32_t)(2 * code_buf + values) * kCodes + kWaveRows * wave * d + 16 * kActive * k + 16 * (lane % kActive);
        raw = lds_load<u32x4>(raw_at);
        raw_at = lds0 + (uint32_t)(values ? kKeyBufs + value_buf : key_buf) * kBuf + piece_at(values, k);
      } else if (kActive == kWave || lane < kActive) {
        if (values && part_of == 1 && t + 1 < n && (t + 1 < whole0 || t + 1 >= whole1) && unseen(t + 1, k)) raw = (u32x4){0u, 0u, 0u, 0u};
        if (part_of == 1) store_half(raw_at, raw[0], raw[1], scale);
        else store_half(raw_at ^ 16u, raw[2], raw[3], scale);
      }
      return;
    }
    if (i == 6 * kLoads) place();
    stage(i - 6 * kLoads);
    if (i == kChores - 1) {
      code_buf = code_buf + 1 == kCodeBufs ? 0 : code_buf + 1;
      key_buf = key_buf + 1 == kKeyBufs ? 0 : key_buf + 1;
      value_buf ^= 1;
    }
  };
  auto chores = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kChores; ++i) chore(t, i);
  };
  // Opens a step: what the step before stored is there for every wave, and the wave's codes of this one's pair have arrived.
  int steps = 0;
  auto arrive = [&]() __attribute__((always_inline)) {
    ++steps;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    wait_loads<2 * kLoads * (kCodeBufs - 1)>();
  };

  const float inv_scale = 1.f / a.scale_log2;
  float l = 0.f, shift = 0.f, limit = -INFINITY;
  f32x16 o[ND];
#pragma unroll
  for (int c = 0; c < ND; ++c) o[c] = (f32x16){};

  // Operands as in k_paged_chunk: tokens 32 (i % NK) .., channels 16 (i / NK) .. of the scores; channels 32 (i % ND) .., tokens
  // 16 (i / ND) .. of the outputs, k slot 8 half + i being token 8 (i / 4) + 4 half + i % 4.
  constexpr int kS = NK * NC, kO = 2 * NK * ND, kAhead = 3;
  constexpr int kEvery = kS >= 2 * kChores ? 2 : 1;  // products of X from one chore to the next (the others come with Y's)
  const uint32_t kaddr = lds0 + r32 * kRow + 16u * (half ^ swizzle_k<T>(r32));
  const uint32_t vrow = 4 * half + (lane % 16) / 4;
  const uint32_t vaddr = lds0 + kKeyBufs * kBuf + vrow * kRow + 16u * ((((lane / 16) & 1) * 2 + (lane % 4) / 2) ^ swizzle_v<T>(vrow)) + 8 * (lane & 1);
  auto load_k = [&](uint32_t x, int i) __attribute__((always_inline)) { return lds_load<u32x4>((x ^ (32u * (i / NK))) + 32 * (i % NK) * kRow); };
  auto load_v = [&](uint32_t x, int i) __attribute__((always_inline)) {
    const uint32_t y = (x ^ (64u * (i % ND))) + 16 * (i / ND) * kRow;
    const u32x2 lo = lds_load_tr(y), hi = lds_load_tr(y + 8 * kRow);
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
  // A tile's probabilities (in place of the scores), rounded to the type once; the sum is that of the rounded ones.
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
    asm volatile("" : "+v"(kat), "+v"(vat));
#pragma unroll
    for (int i = 0; i < kS; ++i) {
      sn[i % NK] = mfma32<BF16>(kf[i % kAhead], qb[i / NK], i < NK ? (f32x16){} : sn[i % NK]);
      if (i % kEvery == 0 && i / kEvery < kChores) chore(t, i / kEvery);
      if (i + kAhead < kS) kf[i % kAhead] = load_k(kat, i + kAhead);
      else vf[i + kAhead - kS] = load_v(vat, i + kAhead - kS);
      __builtin_amdgcn_sched_barrier(0);
    }
    weights(s);
    kr = kr + 1 == kKeyBufs ? 0 : kr + 1;
    vr ^= 1;
    uint32_t knext = kaddr + (uint32_t)kr * kBuf;
    asm volatile("" : "+v"(vat), "+v"(knext));
#pragma unroll
    for (int i = 0; i < kO; ++i) {
      o[i % ND] = mfma32<BF16>(vf[i % kAhead], pb[i / ND], o[i % ND]);
      if (kS / kEvery + i < kChores) chore(t, kS / kEvery + i);
      if (i + kAhead < kO) vf[i % kAhead] = load_v(vat, i + kAhead);
      else kf[i + kAhead - kO] = load_k(knext, i + kAhead - kO);
      __builtin_amdgcn_sched_barrier(0);
    }
    settle(t + 1, sn);
  };
  static_assert(kChores <= kS / kEvery + kO, "a step's chores");
  // The wave's last step.
  auto finish = [&](int t, f32x16 (&s)[NK]) __attribute__((always_inline)) {
    arrive();
    chores(t);
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
    // q, the keys of tiles 0 to 2, the values of tile 0, then pairs 0 to 2: all under way at once.
    u32x4 first[4][kLoads];
    float first_scale[4];
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      place();
#pragma unroll
      for (int v = 0; v <= (t == 0); ++v) {
        first_scale[v ? 3 : t] = scale_of(v ? v_bytes : k_bytes, 0);
        const unsigned char* base = reinterpret_cast<const unsigned char*>(v ? p.v : p.k) + at[0];
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
          if (kActive == kWave || lane < kActive) first[v ? 3 : t][k] = *reinterpret_cast<const u32x4*>(base + (lane_off + kRowsPerLoad * k * row_bytes));
      }
    }
    {
      const uint16_t* q = a.q + (int64_t)(rt.tok0 + my_tok) * a.q_stride + (h * a.G + my_row - my_tok * a.G) * d + 8 * half;
#pragma unroll
      for (int c = 0; c < NC; ++c) qb[c] = *reinterpret_cast<const u32x4*>(q + 16 * c);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kCodeBufs; ++i) {
      place();
#pragma unroll
      for (int k = 0; k < 2 * kLoads; ++k) stage(k);
      code_buf = code_buf + 1 == kCodeBufs ? 0 : code_buf + 1;
    }
    // (q's wait is here: inside the loop it would be one for the tiles' loads too)
    wait_loads<0>();
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(qb[c]));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < kLoads; ++k)
        if (kActive == kWave || lane < kActive) {
          u32x4 x = first[i][k];
          if (i == 3 && (whole0 > 0 || whole1 <= 0) && unseen(0, k)) x = (u32x4){0u, 0u, 0u, 0u};
          const uint32_t dst = lds0 + (uint32_t)i * kBuf + piece_at(i == 3, k);
          store_half(dst, x[0], x[1], first_scale[i]);
          store_half(dst ^ 16u, x[2], x[3], first_scale[i]);
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
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
        finish(t + 1, s1);
      } else {
        finish(t, s0);
      }
    }
    // Steps of the other waves; none may end while its loads are under way.
    while (steps < n) {
      arrive();
      chores(steps - 1);
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
    redo_rows<T, BF16>(a, Pages8<INT8>{a}, part, rt, h, wrow, 32, tl, t0, t0 + n,
                       [&](int r) { return split * part.rows + part_row(a, part, rt, h, r); }, BN);
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
// k_paged8_rows: at most 16 rows, one wave: single tokens (and few) over a long cache.
//
// The codes arrive in LDS, two or three tiles of it at once and for this wave alone, so that there is no barrier: 16 bytes a lane where
// the lane reads them again as the two operands of 8 channels that they are (keys: row l % 16, channels 64 c + 16 (l / 16); the order
// of a product's channels is free as long as q has the same), and rows of values whose pieces are exchanged so that the
// transposing reads, 16 channels of eight tokens, find them in different banks. A lane gets eight tokens' codes of one channel; they
// become values of the type, with their block's power of two, in registers. (Loads to registers, a tile or two ahead: the
// compiler copies registers in flight from one turn to the next, so that each turn waits for all loads: 1.36 us a tile of 64
// tokens at d = 64 for 0.96.) The probabilities meet the values in two parts of the type: errors are an output's own rounding's.
//
// 2 d bytes a token and head bound it, once the waves are busy as long: 16 requests of up to 16384 tokens with 8 kv-heads of 128
// (317 MB, int8) take 62 us, 5.1 TB/s; 16 of 16384 (537 MB, e4m3) 89.5 with the join, 6.0. One wave a SIMD: its vector
// instructions are 42% of its time there, its waits 37%. A single request of 4096 tokens with 32 kv-heads (34 MB) takes 11 to 13 us and
// the join 4: the chain length, page, codes, products twice, and two launches. Loads past the caches, which hold nothing that is read
// twice: 92 us for 105 at 537 MB. Two waves a SIMD: the ragged batch 85 us for 68 with the join, the even one 108 for 89, 4 requests at
// d = 256 32 for 24.5, the single one 18.8 for 15.4; one wave for two of them: 118, 127, 23.7 and 16.9. Four groups of 16 tokens a tile at
// d = 128, or the scores of a tile between the outputs of the one before: nothing gained. Ranges shared out by what the requests see:
// the ragged batch 85 to 68 us; where ranges are short, finding them costs 2 us (17.5 to 19.5 for a window of 1024 tokens), hence
// kFlat8Tokens.
// ------------------------------------------------------------------------------------------
template <int T>
constexpr int rows8_groups() { return T == 1 ? 4 : 2; }  // of 16 tokens, a tile
template <int T>
constexpr int rows8_ring() { return T == 2 ? 3 : 2; }    // tiles in LDS

// A range of a tile of rows: `split` of `splits`.
struct Unit {
  RowTile rt;
  int split, splits;
  uint32_t first;  // where ranges are shared out: the range of the launch that the tile's first one is
};

// Range f of a launch of so many ranges of every tile of rows. Up to 64 requests' tiles are counted, so that ranges that are none are the
// last ones (spread over the launch they made 1024 waves of 32 requests with 32 heads 177 us for 163), by one round of loads.
__device__ __forceinline__ bool unit_of_splits(const PagedAttnArgs& a, uint32_t f, int splits, Unit& u) {
  const int B = a.p.B, lane = (int)lane_id(), tile = (int)(f / (uint32_t)splits);
  u.split = (int)(f - (uint32_t)tile * (uint32_t)splits);
  u.splits = splits;
  u.first = 0;
  if (B <= kWave) {
    const int b = min(lane, B - 1), cu = a.cu[b], next = a.cu[b + 1], len = a.p.state[b];
    const int rows = (min(next, a.n_q) - cu) * a.G;
    const uint32_t n = lane < B && rows > 0 ? (uint32_t)(rows + kFewRows - 1) / kFewRows : 0u, incl = wave_incl_scan(n);
    const int at = __builtin_popcountll(ballot(incl <= (uint32_t)tile));
    if (at == kWave) return false;
    u.rt = rows_at(a, at, __builtin_amdgcn_readlane(cu, at), __builtin_amdgcn_readlane(next, at), __builtin_amdgcn_readlane(len, at));
    u.rt.row0 = (tile - __builtin_amdgcn_readlane((int)(incl - n), at)) * kFewRows;
    return true;
  }
  u.rt = B <= kCounted ? row_tile<kFewRows>(a, tile, false) : spread_tile<kFewRows>(a, tile);
  return u.rt.row0 < u.rt.rows;
}

// Range f of a launch whose ranges are shared out among the requests by what they see: `chunk` tiles each (at least 64 tokens), evenly
// within a request, as few of them as make no more than a.budget ranges (one a tile of rows, if those are more).
__device__ __forceinline__ bool unit_of(const Paged8AttnArgs& a, uint32_t f, int BN, Unit& u) {
  struct Entry {
    RowTile rt;
    uint32_t tiles, n;  // of rows, and of tokens that they see
  };
  constexpr int kEach = kFlat8Requests / kWave;  // requests of a lane
  constexpr int kHalvings = 2;
  const int B = a.p.B, lane = (int)lane_id(), stride = (B + kWave - 1) / kWave;
  auto entry = [&](int b, bool is) {
    Entry e;
    b = min(b, B - 1);
    const int next = a.cu[b + 1];
    e.rt = rows_at(a, b, a.cu[b], next, a.p.state[b]);
    e.tiles = e.n = 0;
    if (is && e.rt.rows > 0) {
      e.tiles = a.mixed ? e.rt.rows <= kFewRows : (uint32_t)(e.rt.rows + kFewRows - 1) / kFewRows;
      e.n = (uint32_t)TileList(e.rt.base, e.rt.base + min(next, a.n_q) - e.rt.tok0 - 1, a.window, a.sinks, BN).n;
    }
    return e;
  };
  uint32_t tiles[kEach], n[kEach], units = 0;
  uint64_t work = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    tiles[i] = n[i] = 0;
    if (i >= stride) continue;
    const Entry e = entry(lane * stride + i, lane * stride + i < B);
    tiles[i] = e.tiles;
    n[i] = e.n;
    units += e.tiles;
    work += (uint64_t)e.tiles * e.n;
  }
  auto sum = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan(x), kWave - 1); };
  const uint64_t total = sum((uint32_t)(work & 0xffffu)) + ((uint64_t)sum((uint32_t)(work >> 16)) << 16);
  uint32_t chunk = 1, count = 0;
  auto ranges = [&](uint32_t x) { return max((x + chunk - 1) / chunk, 1u); };
  auto divide = [&](uint32_t by) {
    chunk = total < 0x80000000u ? ((uint32_t)total + by - 1) / by : (uint32_t)min(total / by + 1, (uint64_t)0x7fffffff);
    chunk = max(chunk, (uint32_t)(kWave / BN));
    count = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (i < stride) count += tiles[i] * ranges(n[i]);
  };
  // Each request's last range may be a part of one. Where that makes too many, one for each is kept back at most, and fewer where
  // they do: by halves, 71.3 us to 69.0 for 16 ragged requests (more than two halvings find less than they take).
  const uint32_t budget = (uint32_t)a.budget;
  divide(budget);
  if (sum(count) > budget) {
    uint32_t least = budget - min(sum(units), budget - 1), most = budget;
#pragma unroll 1
    for (int i = 0; i < kHalvings; ++i) {
      const uint32_t by = (least + most) / 2;
      divide(by);
      if (sum(count) > budget) most = by;
      else least = by;
    }
    divide(least);
  }
  uint32_t incl = wave_incl_scan(count), want = f;
  if (want >= (uint32_t)__builtin_amdgcn_readlane((int)incl, kWave - 1)) return false;
  int at = __builtin_popcountll(ballot(incl <= want)), b = at;
  want -= (uint32_t)__builtin_amdgcn_readlane((int)(incl - count), at);
  uint32_t each = ranges(n[0]);
  if (stride > 1) {
    b *= stride;
    const Entry e = entry(b + lane, lane < stride && b + lane < B);
    each = ranges(e.n);
    count = e.tiles * each;
    incl = wave_incl_scan(count);
    at = __builtin_popcountll(ballot(incl <= want));
    want -= (uint32_t)__builtin_amdgcn_readlane((int)(incl - count), at);
    b += at;
  }
  u.rt = rows_of(a, b);
  u.splits = __builtin_amdgcn_readlane((int)each, at);
  const int row_tile = (int)(want / (uint32_t)u.splits);
  u.rt.row0 = row_tile * kFewRows;
  u.split = (int)want - row_tile * u.splits;
  u.first = f - (uint32_t)u.split;
  return true;
}

// Four direct loads of 16 bytes a lane to dst, dst + 1024, .. (m0, their LDS address, is put back; five cycles lie between a base
// that the vector units wrote and its use, one between m0 and its). What the wave has read of the place before is there.
__device__ __forceinline__ void load_4_to_lds(uint32_t dst, const unsigned char* b0, uint32_t o0, const unsigned char* b1, uint32_t o1,
                                              const unsigned char* b2, uint32_t o2, const unsigned char* b3, uint32_t o3) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_waitcnt lgkmcnt(0)\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %2, %6 nt\n\t"
               "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %7 nt\n\t"
               "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %8 nt\n\t"
               "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %9 nt\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(dst), "v"(o0), "v"(o1), "v"(o2), "v"(o3), "s"(b0), "s"(b1), "s"(b2), "s"(b3) : "memory", "scc");
}

template <int T, bool BF16, bool INT8>
__global__ __launch_bounds__(kWave) void k_paged8_rows(Paged8AttnArgs a, PartOut part) {
  constexpr int d = kTile * T, NC = 2 * T, NO = 4 * T, NG = rows8_groups<T>(), BN = 16 * NG, R = rows8_ring<T>();
  constexpr int kLanes = 4 * T, kRowsPerLoad = 16 / T;             // of a row of values, of a load of them
  constexpr int kLoads = NG * T;                                   // of a tile's keys, and of its values
  // int8 codes become whole numbers of the type without their scale, which multiplies the scores and, in bf16, whose exponents have
  // room for it, the probabilities: fewer instructions than to multiply them.
  constexpr bool kScaled = INT8 && BF16;
  // Such sums of codes leave fp32 for queries of 2^113 and more, and one of -inf is a weight of 0 whatever the score. Rows with a query
  // whose square leaves it, of 2^64 and more, are done by themselves, with keys that have their scale.
  bool beyond = false;
  constexpr uint32_t kHalf = 1024 * kLoads, kSlot = 2 * kHalf;     // bytes of each, of a tile
  __shared__ __align__(1024) unsigned char smem[R * kSlot];
  const PagedView& p = a.p;
  const int h = blockIdx.x % p.H;
  Unit u;
  if (a.flat) {
    if (!unit_of(a, blockIdx.x / p.H, BN, u)) return;
  } else if (!a.mixed) {
    if (!unit_of_splits(a, blockIdx.x / p.H, part.n_splits, u)) return;
  } else {
    u.split = (blockIdx.x / p.H) % part.n_splits;
    u.splits = part.n_splits;
    u.rt = rows_of(a, blockIdx.x / (p.H * part.n_splits));
    if (u.rt.rows <= 0 || u.rt.rows > kFewRows) return;
  }
  const RowTile rt = u.rt;
  // Where the results of row r of the request go if they are a range's.
  auto result_at = [&](int r) __attribute__((always_inline)) {
    if (a.flat) return ((int64_t)(u.first + (uint32_t)u.split) * p.H + h) * kFewRows + (r - rt.row0);
    return u.split * part.rows + part_row(a, part, rt, h, r);
  };
  const uint32_t lane = lane_id(), r16 = lane % 16, q4 = lane / 16;
  const int row = min(rt.row0 + (int)r16, rt.rows - 1), tok = row / a.G, pos = rt.base + tok;
  const int pos0 = rt.base + rt.row0 / a.G, pos1 = rt.base + (min(rt.row0 + kFewRows, rt.rows) - 1) / a.G;
  const TileList tl(pos0, pos1, a.window, a.sinks, BN);
  const int t0 = range_start(tl.n, u.split, u.splits), n = range_start(tl.n, u.split + 1, u.splits) - t0;
  // Where its ranges' results begin and how many there are, for each row.
  if (a.flat && u.split == 0 && q4 == 0 && rt.row0 + (int)r16 < rt.rows)
    a.info[part_row(a, part, rt, h, row)] = make_int2((int)result_at(row), u.splits);
  // Tiles [clean0, clean1) are seen whole by every row, [whole0, whole1) by some.
  const int clean0 = a.window > 0 ? tl.count_to(before(pos1, a.window), BN) - t0 : 0, clean1 = tl.count_to(pos0 - BN + 1, BN) - t0;
  const int whole0 = tl.count_to(tl.lo - 1, BN) - t0, whole1 = tl.count_to(tl.hi - BN + 1, BN) - t0;

  // Lane i holds the offset in k and v, and the scales, of group i of 16 tokens of the 64 / NG tiles whose loads are next (one that
  // no row sees is replaced by the nearest that some row does; pages hold 16 tokens or more, and so do blocks).
  constexpr int kBatch = kWave / NG;
  static_assert(R <= kBatch, "tiles under way are of two batches at most");
  uint32_t at_lo = 0, at_hi = 0, scales = 0, scales_before = 0;
  auto look_up = [&](int first) __attribute__((always_inline)) {
    const int j = tl.start(t0 + min(first + (int)lane / NG, n - 1), BN) + 16 * ((int)lane % NG);
    const int g0 = j < tl.sinks ? j : min(max(j, tl.lo & ~15), tl.hi & ~15);
    int page = p.table[(int64_t)rt.b * p.max_pages + (g0 >> p.log2_page)];
    if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
    const int place = g0 & ((1 << p.log2_page) - 1);
    const int64_t at = (int64_t)page * p.page_stride + (int64_t)h * p.head_stride + (int64_t)place * p.token_stride;
    const int64_t block = (((int64_t)page * p.H + h) << (p.log2_page - a.log2_block)) + (place >> a.log2_block);
    at_lo = (uint32_t)at;
    at_hi = (uint32_t)(at >> 32);
    scales_before = scales;
    scales = (uint32_t)a.k_scale[block] | (uint32_t)a.v_scale[block] << 8;
  };
  // Loads: the lane's place in a group's keys, and its row of values and piece of it (rows of the two groups of a product's tokens
  // lie in different banks, and so do four rows from a fourth one on).
  const uint32_t lds0 = (uint32_t)(uintptr_t)smem, row_bytes = (uint32_t)p.token_stride;
  const uint32_t k_off = r16 * row_bytes + 16u * q4, v_row = lane / kLanes;
  auto exchanged = [&](uint32_t row_of_group, uint32_t group) __attribute__((always_inline)) {
    return (T == 4 ? row_of_group & 3 : T == 2 ? row_of_group >> 1 & 1 : 0u) | (group & 1) * T;
  };
  uint32_t v_off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) v_off[i] = v_row * row_bytes + 16u * ((lane % kLanes) ^ exchanged(v_row, i));
  const unsigned char *const k0 = reinterpret_cast<const unsigned char*>(p.k), *const v0 = reinterpret_cast<const unsigned char*>(p.v);
  auto stage = [&](int t, int slot) __attribute__((always_inline)) {
    if (t % kBatch == 0) look_up(t);
    uint64_t at[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int i = (NG * t + g) % kWave;
      at[g] = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at_hi, i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)at_lo, i);
    }
    const uint32_t dst = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds0 + (uint32_t)slot * kSlot));
#pragma unroll
    for (int l = 0; l < kLoads; l += 4) {
      // keys: load l is channels 64 (l % T) .. of group l / T
      auto key = [&](int i) __attribute__((always_inline)) { return k0 + at[i / T] + 64 * (i % T); };
      load_4_to_lds(dst + 1024 * l, key(l), k_off, key(l + 1), k_off, key(l + 2), k_off, key(l + 3), k_off);
    }
#pragma unroll
    for (int l = 0; l < kLoads; l += 4) {
      // values: rows kRowsPerLoad (l % T) .. of it
      auto value = [&](int i) __attribute__((always_inline)) { return v0 + at[i / T] + (uint64_t)(kRowsPerLoad * (i % T)) * row_bytes; };
      load_4_to_lds(dst + kHalf + 1024 * l, value(l), v_off[l / T % 2], value(l + 1), v_off[(l + 1) / T % 2], value(l + 2), v_off[(l + 2) / T % 2],
                    value(l + 3), v_off[(l + 3) / T % 2]);
    }
  };
  // What no row sees of a tile's values is cleared: it may be what memory held, and 0 times NaN is not 0 (int8 has none, and a
  // block with a token that is seen has its scale; the scores of such keys are replaced).
  auto clear_values = [&](int t, uint32_t slot_at) __attribute__((always_inline)) {
    if (INT8 || (t >= whole0 && t < whole1)) return;
    const int j0 = tl.start(t0 + t, BN) + (int)v_row;
#pragma unroll 1
    for (int l = 0; l < kLoads; ++l) {
      const int j = j0 + kRowsPerLoad * l;
      if (j > tl.hi || (j < tl.lo && j >= tl.sinks))
        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(slot_at + kHalf + 1024 * l + 16 * lane) = (u32x4){0u, 0u, 0u, 0u};
    }
    asm volatile("" ::: "memory");
  };
  // Lanes 2 i and 2 i + 1 of 16 address the row of token i of their product's eight: 4 (l / 16) .. of its first group, then its second.
  const uint32_t read_row = 4 * q4 + r16 / 2 % 4, read_group = r16 / 8;
  const uint32_t read_at = (16 * read_group + read_row) * d + 8 * (r16 & 1), read_x = exchanged(read_row, read_group);
  auto values_at = [&](uint32_t slot_at, int c, int g) __attribute__((always_inline)) {  // channels 16 c .., of groups g and g + 1
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const uint32_t x = slot_at + kHalf + 16 * g * d + read_at + 16u * ((uint32_t)c ^ read_x);
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<__attribute__((address_space(3))) i32x2*>(x)));
  };

  const float inv_scale = 1.f / a.scale_log2;
  float l = 0.f, shift = 0.f, limit = -INFINITY;
  f32x4 o[NO];  // rows 4 (l / 16) + e, channel 16 c + l % 16
#pragma unroll
  for (int c = 0; c < NO; ++c) o[c] = (f32x4){};
  if (n > 0) {
    u32x4 qb[NC];  // Q as the B operand: column = row, k = 64 (c / 2) + 16 (l / 16) + 8 (c % 2) + i
    {
      const uint16_t* q = a.q + (int64_t)(rt.tok0 + tok) * a.q_stride + (h * a.G + row - tok * a.G) * d + 16 * q4;
#pragma unroll
      for (int c = 0; c < NC; ++c) qb[c] = *reinterpret_cast<const u32x4*>(q + 64 * (c / 2) + 8 * (c % 2));
    }
    // The scale bytes of group g of tile t, whose batch of tiles is that of the newest one that is placed, `newest`, or the one before.
    auto scale_bytes = [&](int t, int newest, int g) __attribute__((always_inline)) {
      const uint32_t word = t / kBatch == newest / kBatch ? scales : scales_before;
      return (uint32_t)__builtin_amdgcn_readlane((int)word, (NG * t + g) % kWave);
    };
    auto scores = [&](int t, int newest, uint32_t slot_at, f32x4 (&s)[NG]) __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const float scale = power_of(scale_bytes(t, newest, g) & 0xffu);
        s[g] = (f32x4){};
#pragma unroll
        for (int c = 0; c < T; ++c) {
          const u32x4 k = lds_load<u32x4>(slot_at + 1024 * (g * T + c) + 16 * lane);
          u32x2 x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = INT8 ? whole_pairs<BF16>(k[i]) : decode_pairs<BF16, false>(k[i], scale);
          s[g] = mfma16<BF16>((u32x4){x[0].x, x[0].y, x[1].x, x[1].y}, qb[2 * c], s[g]);
          s[g] = mfma16<BF16>((u32x4){x[2].x, x[2].y, x[3].x, x[3].y}, qb[2 * c + 1], s[g]);
        }
        if constexpr (INT8) s[g] *= scale;
      }
    };
    // The scores of tile t are masked and the shift follows them.
    auto settle = [&](int t, f32x4 (&s)[NG]) __attribute__((always_inline)) {
      if (t < clean0 || t >= clean1) {
        const int j0 = tl.start(t0 + t, BN) + 4 * (int)q4;
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!sees(pos, j0 + 16 * g + e, a.window, a.sinks)) s[g][e] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int e = 1; e < 4 * NG; ++e) top = fmaxf(top, s[e / 4][e % 4]);
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
    };
    // Tile t's probabilities, in two parts of the type, the second what the first leaves, and their products with its values.
    auto outputs = [&](int t, int newest, uint32_t slot_at, const f32x4 (&s)[NG]) __attribute__((always_inline)) {
      u32x4 pa[NG / 2], pl[NG / 2];
      float vs[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) vs[g] = power_of(scale_bytes(t, newest, g) >> 8 & 0xffu);
#pragma unroll
      for (int e = 0; e < 2 * NG; ++e) {
        float x = __builtin_amdgcn_exp2f(fmaf(s[e / 2][2 * (e % 2)], a.scale_log2, shift));
        float y = __builtin_amdgcn_exp2f(fmaf(s[e / 2][2 * (e % 2) + 1], a.scale_log2, shift));
        l += x + y;
        if (kScaled) x *= vs[e / 2], y *= vs[e / 2];
        pa[e / 4][e % 4] = pack2<BF16>(x, y);
        pl[e / 4][e % 4] = pack2<BF16>(x - to_float<BF16>(pa[e / 4][e % 4] & 0xffffu), y - to_float<BF16>(pa[e / 4][e % 4] >> 16));
      }
#pragma unroll
      for (int g = 0; g < NG; g += 2)
#pragma unroll
        for (int c = 0; c < NO; ++c) {
          const u32x2 w = values_at(slot_at, c, g);
          const u32x2 x = kScaled ? whole_pairs<BF16>(w.x) : decode_pairs<BF16, INT8>(w.x, vs[g]);
          const u32x2 y = kScaled ? whole_pairs<BF16>(w.y) : decode_pairs<BF16, INT8>(w.y, vs[g + 1]);
          const u32x4 v = {x.x, x.y, y.x, y.y};
          o[c] = mfma16<BF16>(pl[g / 2], v, mfma16<BF16>(pa[g / 2], v, o[c]));
        }
    };
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i < n) stage(i, i);
    if constexpr (kScaled) {
      // (the first tiles are under way)
      float squares[2] = {};
#pragma unroll
      for (int i = 0; i < 4 * NC; ++i) {
        const uint32_t pair = qb[i / 4][i % 4];
        const bf16x2 x = __builtin_bit_cast(bf16x2, pair);
        squares[i % 2] = __builtin_amdgcn_fdot2_f32_bf16(x, x, squares[i % 2], false);
      }
      beyond = !(squares[0] + squares[1] < INFINITY);
    }
    int slot = 0;
    for (int t = 0; t < n; ++t) {
      // The tile's loads have arrived; those of the tiles behind it are under way.
      if (t + R <= n) wait_loads<2 * kLoads * (R - 1)>();
      else wait_loads<0>();
      const uint32_t slot_at = lds0 + (uint32_t)slot * kSlot;
      const int newest = min(t + R, n) - 1;
      f32x4 s[NG];
      scores(t, newest, slot_at, s);
      settle(t, s);
      clear_values(t, slot_at);
      outputs(t, newest, slot_at, s);
      if (t + R < n) stage(t + R, slot);
      slot = slot + 1 == R ? 0 : slot + 1;
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
  if (ballot(z != z || (rt.row0 + (int)r16 < rt.rows && (beyond || fabsf(shift) >= kFar<BF16>)))) {
    redo_rows<T, BF16>(a, Pages8<INT8>{a}, part, rt, h, rt.row0, kFewRows, tl, t0, t0 + n, result_at, BN);
    return;
  }
  if (part.n_splits > 1 && q4 == 0 && rt.row0 + (int)r16 < rt.rows) {
    part.ml[result_at(row)] = make_float2(limit > -INFINITY ? -shift : -INFINITY, pos < 0 ? -1.f : l);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int orow = rt.row0 + (int)(4 * q4) + e, otok = orow / a.G, hq = h * a.G + orow - otok * a.G;
    const float le = __shfl(l, (int)(4 * q4) + e, kWave);
    if (orow >= rt.rows) continue;
    const int64_t t = rt.tok0 + otok;
    if (part.n_splits > 1) {
      float* dst = part.o + result_at(orow) * d + r16;
#pragma unroll
      for (int c = 0; c < NO; ++c) dst[16 * c] = o[c][e];
    } else {
      const float inv = rt.base + otok < 0 ? 0.f : 1.f / le;
      uint16_t* dst = a.out + t * a.out_stride + hq * d + r16;
#pragma unroll
      for (int c = 0; c < NO; ++c) dst[16 * c] = (uint16_t)pack2<BF16>(o[c][e] * inv, 0.f);
    }
  }
}

// ------------------------------------------------------------------------------------------
// k_paged8_merge: joins the ranges of a row where requests have different numbers of them. As k_paged_merge: sum of 2^(m_i - m) l_i and
// of the outputs so weighted. 64 rows of 16 requests take 4.6 us, latencies (a row's place, its ranges' sums, their outputs).
// ------------------------------------------------------------------------------------------
template <int T, bool BF16, int OF, bool WIDE>
__global__ __launch_bounds__(kMergeThreads) void k_paged8_merge(Paged8AttnArgs a, PartOut part) {
  constexpr int L = 16 * T, S = kMergeThreads / L;
  const int64_t i0 = WIDE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * S + (int)threadIdx.x / L;
  int t, hq;
  int2 info = make_int2(0, 0);
  bool mine;
  if (a.mixed) {  // row r of an entry and kv-head
    const int r = (int)(i0 % kFewRows), h = (int)(i0 / kFewRows % a.p.H), b = (int)(i0 / kFewRows / a.p.H);
    if (b >= a.p.B) return;
    const RowTile rt = rows_of(a, b);  // (a wave's rows are one request's: S divides kFewRows)
    mine = r < rt.rows && rt.rows <= kFewRows;
    t = rt.tok0 + r / a.G;
    hq = h * a.G + r % a.G;
    if (mine) info = a.info[part.by_entry ? i0 : (int64_t)t * a.Hq + hq];
  } else {
    t = (int)(i0 / a.Hq);
    hq = (int)(i0 - (int64_t)t * a.Hq);
    if (i0 >= (int64_t)a.n_q * a.Hq) return;
    info = a.info[i0];  // (of a row of a request if it is one)
    mine = t < a.cu[a.p.B];
  }
  if (!mine) return;  // (all of a stream; WIDE: all of the workgroup)
  // (starts that are none, not ascending, have rows that no range is of: what memory held is not read for an address)
  const int64_t step = (int64_t)a.p.H * kFewRows;
  if (info.x < 0 || info.y < 1 || info.x + (info.y - 1) * step >= a.flat * step) return;
  merge_row<T, BF16, OF, WIDE>(a, part.ml, part.o, step, info.y, info.x, t, hq);
}

template <int T, bool BF16>
static hipError_t merge8_launch(const Paged8AttnArgs& a, const PartOut& part, hipStream_t s) {
  const int64_t rows = a.mixed ? (int64_t)a.p.B * a.p.H * kFewRows : (int64_t)a.n_q * a.Hq;
  if (rows >= kMergeWideRows)
    hipLaunchKernelGGL((k_paged8_merge<T, BF16, 16 * T, false>), dim3((uint32_t)merge_groups(rows, T)), dim3(kMergeThreads), 0, s, a, part);
  else
    hipLaunchKernelGGL((k_paged8_merge<T, BF16, kWave, true>), dim3((uint32_t)rows), dim3(kMergeThreads), 0, s, a, part);
  return hipGetLastError();
}

template <int T, bool BF16, bool INT8>
static hipError_t attn8_launch(Paged8AttnArgs a, hipStream_t s) {
  // (all outputs first, aligned as they are accessed)
  const int64_t rows = (int64_t)a.n_q * a.Hq, n_few = paged8_parts(a, a.few_rows), n_many = paged_parts(rows, a.many);
  float* const o = (float*)a.ws;
  float2* const ml = (float2*)(o + (n_few + n_many) * (64 * T));
  a.info = (int2*)(ml + n_few + n_many);
  const PartOut few = {ml, o, a.few_rows, a.by_entry, a.few}, many = {ml + n_few, o + n_few * (64 * T), rows, 0, a.many};
  hipError_t e;
  if (a.few > 0) {
    const int64_t ranges = a.flat ? a.flat : (a.mixed ? a.p.B : paged_tiles(a.p, a.G, a.n_q, kFewRows)) * a.few;
    hipLaunchKernelGGL((k_paged8_rows<T, BF16, INT8>), dim3((uint32_t)(ranges * a.p.H)), dim3(kWave), 0, s, a, few);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.many > 0) {
    const int64_t tiles = paged_tiles(a.p, a.G, a.n_q, chunk_rows(T));
    hipLaunchKernelGGL((k_paged8_chunk<T, BF16, INT8>), dim3((uint32_t)(tiles * a.p.H * a.many)), dim3(kWave * chunk_waves(T)), 0, s,
                       a, many);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if ((e = a.flat ? merge8_launch<T, BF16>(a, few, s) : launch_paged_merge(a, few, true, s)) != hipSuccess) return e;
  return launch_paged_merge(a, many, false, s);
}

template <int T>
static hipError_t attn8_of_types(const Paged8AttnArgs& a, hipStream_t s) {
  if (a.int8) return a.p.bf16 ? attn8_launch<T, true, true>(a, s) : attn8_launch<T, false, true>(a, s);
  return a.p.bf16 ? attn8_launch<T, true, false>(a, s) : attn8_launch<T, false, false>(a, s);
}

hipError_t launch_paged8_attn(const Paged8AttnArgs& a, hipStream_t s) {
  switch (a.p.d) {
    case 64: return attn8_of_types<1>(a, s);
    case 128: return attn8_of_types<2>(a, s);
    default: return attn8_of_types<4>(a, s);
  }
}

}  // namespace mf
