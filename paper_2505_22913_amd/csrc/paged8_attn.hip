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

// ------------------------------------------------------------------------------------------
// k_paged8_chunk: 32 rows a wave, 8 waves a workgroup (4 at d = 256), tiles of 64 tokens (32): chunks of prompts.
//
// The products are k_paged_chunk's, over tiles of values in LDS. Codes become values once a workgroup: a tile's codes arrive in LDS
// by direct loads, three steps ahead, each wave converts the rows that it has loaded itself (so their arrival needs no
// barrier) and stores them where the products read them; the step's one barrier hands them to the others. Pair p is the codes
// of the keys of tile p + 3 and of the values of tile p + 1; step t converts pair t, a piece at a time between the products, and
// loads pair t + 3 in its place. So three buffers of keys do (one that X reads, the next one, whose first operands are read before
// the barrier, and the one that is written) and two of values.
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
    redo_rows<T, BF16>(a, Pages8<INT8>{a}, part, rt, h, wrow, 32, tl, t0, t0 + n, split, BN);
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
// k_paged8_rows: at most 16 rows, one wave, tiles of 32 tokens.
//
// As k_paged_rows: the products' operands come straight from memory. A lane loads 16 codes of a key row at once, channels
// 64 c + 16 (l / 16), which are two operands of 8 channels each (the order of a product's channels is free as long as q
// has the same); of the values it loads channels 4 T (l % 16) .. of eight tokens and transposes them, a byte permute for two codes,
// before they become values of the type. The scale goes into that conversion.
// ------------------------------------------------------------------------------------------
constexpr int kRows8Tile = 32;

template <int T, bool BF16, bool INT8>
__global__ __launch_bounds__(kWave) void k_paged8_rows(Paged8AttnArgs a, PartOut part) {
  constexpr int d = kTile * T, NC = 2 * T, NO = 4 * T, BN = kRows8Tile;
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

  // Lane i holds the offset in k and v, and the scales, of group i of 16 tokens of the 32 tiles at hand (one that no row sees is
  // replaced by the nearest that some row does; pages hold 16 tokens or more, and so do blocks).
  uint32_t at_lo = 0, at_hi = 0, scales = 0;
  const uint32_t row_bytes = (uint32_t)p.token_stride;
  auto group_of = [&](int t, int g) __attribute__((always_inline)) {
    const int g0 = tl.start(t0 + t, BN) + 16 * g;
    return g0 < tl.sinks ? g0 : min(max(g0, tl.lo & ~15), tl.hi & ~15);
  };
  auto look_up = [&](int first) __attribute__((always_inline)) {
    const int g0 = group_of(min(first + (int)lane / 2, n - 1), lane & 1);
    int page = p.table[(int64_t)rt.b * p.max_pages + (g0 >> p.log2_page)];
    if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
    const int place = g0 & ((1 << p.log2_page) - 1);
    const int64_t at = (int64_t)page * p.page_stride + (int64_t)h * p.head_stride + (int64_t)place * p.token_stride;
    const int64_t block = (((int64_t)page * p.H + h) << (p.log2_page - a.log2_block)) + (place >> a.log2_block);
    at_lo = (uint32_t)at;
    at_hi = (uint32_t)(at >> 32);
    scales = (uint32_t)a.k_scale[block] | (uint32_t)a.v_scale[block] << 8;
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
  u32x4 kr[2][T];
  uint32_t vr[8][T];
  float ks[2], vs[2];  // of the tile whose codes are loaded
  auto load_keys = [&](int t) __attribute__((always_inline)) {
    if (t % (kWave / 2) == 0) look_up(t);
    const bool edge = t < whole0 || t >= whole1;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t r = r16;
      if (edge) r = (uint32_t)nearest((int)r, t, g);
      const unsigned char* x = base_of(p.k, t, g) + (r * row_bytes + 16u * q4);
#pragma unroll
      for (int c = 0; c < T; ++c) kr[g][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x + 64 * c));
      ks[g] = power_of((uint32_t)__builtin_amdgcn_readlane((int)scales, (2 * t + g) % kWave) & 0xffu);
    }
  };
  auto load_values = [&](int t) __attribute__((always_inline)) {
    const bool edge = t < whole0 || t >= whole1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t r = 4 * q4 + i % 4;
      if (edge) r = (uint32_t)nearest((int)r, t, i / 4);
      const unsigned char* x = base_of(p.v, t, i / 4) + (r * row_bytes + (uint32_t)NO * r16);
      if constexpr (T == 1) {
        vr[i][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(x));
      } else if constexpr (T == 2) {
        const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(x));
        vr[i][0] = v.x;
        vr[i][1] = v.y;
      } else {
        const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x));
#pragma unroll
        for (int m = 0; m < 4; ++m) vr[i][m] = v[m];
      }
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) vs[g] = power_of((uint32_t)__builtin_amdgcn_readlane((int)scales, (2 * t + g) % kWave) >> 8 & 0xffu);
  };

  const float inv_scale = 1.f / a.scale_log2;
  float l = 0.f, shift = 0.f, limit = -INFINITY;
  f32x4 o[NO];
#pragma unroll
  for (int c = 0; c < NO; ++c) o[c] = (f32x4){};
  if (n > 0) {
    load_keys(0);
    u32x4 qb[NC];  // Q as the B operand: column = row, k = 64 (c / 2) + 16 (l / 16) + 8 (c % 2) + i
    {
      const uint16_t* q = a.q + (int64_t)(rt.tok0 + tok) * a.q_stride + (h * a.G + row - tok * a.G) * d + 16 * q4;
#pragma unroll
      for (int c = 0; c < NC; ++c) qb[c] = *reinterpret_cast<const u32x4*>(q + 64 * (c / 2) + 8 * (c % 2));
    }
    load_values(0);
    for (int t = 0; t < n; ++t) {
      f32x4 s[2] = {};
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const u32x2 lo = decode_pairs<BF16, INT8>(kr[g][c / 2][2 * (c % 2)], ks[g]), hi = decode_pairs<BF16, INT8>(kr[g][c / 2][2 * (c % 2) + 1], ks[g]);
          s[g] = mfma16<BF16>((u32x4){lo.x, lo.y, hi.x, hi.y}, qb[c], s[g]);
        }
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
      for (int m = 0; m < T; ++m) {
        // Channels 4 m .. of the lane's: a word of four tokens for each.
        uint32_t w[2][4];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const uint32_t ab = __builtin_amdgcn_perm(vr[4 * g + 1][m], vr[4 * g][m], 0x05010400u);      // a0 b0 a1 b1
          const uint32_t ab2 = __builtin_amdgcn_perm(vr[4 * g + 1][m], vr[4 * g][m], 0x07030602u);     // a2 b2 a3 b3
          const uint32_t cd = __builtin_amdgcn_perm(vr[4 * g + 3][m], vr[4 * g + 2][m], 0x05010400u);
          const uint32_t cd2 = __builtin_amdgcn_perm(vr[4 * g + 3][m], vr[4 * g + 2][m], 0x07030602u);
          w[g][0] = __builtin_amdgcn_perm(cd, ab, 0x05040100u);
          w[g][1] = __builtin_amdgcn_perm(cd, ab, 0x07060302u);
          w[g][2] = __builtin_amdgcn_perm(cd2, ab2, 0x05040100u);
          w[g][3] = __builtin_amdgcn_perm(cd2, ab2, 0x07060302u);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const u32x2 lo = decode_pairs<BF16, INT8>(w[0][c], vs[0]), hi = decode_pairs<BF16, INT8>(w[1][c], vs[1]);
          const u32x4 v = {lo.x, lo.y, hi.x, hi.y};
          o[4 * m + c] = mfma16<BF16>(pl, v, mfma16<BF16>(pa, v, o[4 * m + c]));
        }
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
    redo_rows<T, BF16>(a, Pages8<INT8>{a}, part, rt, h, rt.row0, kFewRows, tl, t0, t0 + n, split, BN);
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

template <int T, bool BF16, bool INT8>
static hipError_t attn8_launch(const Paged8AttnArgs& a, hipStream_t s) {
  // (all outputs first, aligned as they are accessed)
  const int64_t rows = (int64_t)a.n_q * a.Hq, n_few = paged_parts(a.few_rows, a.few), n_many = paged_parts(rows, a.many);
  float* const o = (float*)a.ws;
  float2* const ml = (float2*)(o + (n_few + n_many) * (64 * T));
  const PartOut few = {ml, o, a.few_rows, a.by_entry, a.few}, many = {ml + n_few, o + n_few * (64 * T), rows, 0, a.many};
  hipError_t e;
  if (a.few > 0) {
    const int64_t tiles = a.mixed ? a.p.B : paged_tiles(a.p, a.G, a.n_q, kFewRows);
    hipLaunchKernelGGL((k_paged8_rows<T, BF16, INT8>), dim3((uint32_t)(tiles * a.p.H * a.few)), dim3(kWave), 0, s, a, few);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.many > 0) {
    const int64_t tiles = paged_tiles(a.p, a.G, a.n_q, chunk_rows(T));
    hipLaunchKernelGGL((k_paged8_chunk<T, BF16, INT8>), dim3((uint32_t)(tiles * a.p.H * a.many)), dim3(kWave * chunk_waves(T)), 0, s,
                       a, many);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if ((e = launch_paged_merge(a, few, true, s)) != hipSuccess) return e;
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
