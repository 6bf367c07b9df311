// Causal attention of the new tokens of every request over its pages (gfx950), with an
// optional sliding window and first tokens that stay visible.
#include <type_traits>

#include "paged_attn.h"

namespace mf {

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
constexpr int kDepth = 3, kRing = kDepth + 1;

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
    redo_rows<T, BF16>(a, Pages16<BF16>{p}, part, rt, h, wrow, 32, tl, t0, t0 + n,
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
    redo_rows<T, BF16>(a, Pages16<BF16>{p}, part, rt, h, rt.row0, kFewRows, tl, t0, t0 + n,
                       [&](int r) { return split * part.rows + part_row(a, part, rt, h, r); }, BN);
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
template <int T, bool BF16, int OF, bool WIDE>
__global__ __launch_bounds__(kMergeThreads) void k_paged_merge(PagedAttnArgs a, PartOut part, int of_few) {
  constexpr int L = 16 * T, S = kMergeThreads / L;
  const int stream = (int)threadIdx.x / L;
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
  merge_row<T, BF16, OF, WIDE>(a, part.ml, part.o, rows, part.n_splits, row, t, hq);
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

hipError_t launch_paged_merge(const PagedAttnArgs& a, const PartOut& part, bool of_few, hipStream_t s) {
  switch (a.p.d) {
    case 64: return a.p.bf16 ? merge_launch<1, true>(a, part, of_few, s) : merge_launch<1, false>(a, part, of_few, s);
    case 128: return a.p.bf16 ? merge_launch<2, true>(a, part, of_few, s) : merge_launch<2, false>(a, part, of_few, s);
    default: return a.p.bf16 ? merge_launch<4, true>(a, part, of_few, s) : merge_launch<4, false>(a, part, of_few, s);
  }
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.p.d) {
    case 64: return a.p.bf16 ? attn_launch<1, true>(a, s) : attn_launch<1, false>(a, s);
    case 128: return a.p.bf16 ? attn_launch<2, true>(a, s) : attn_launch<2, false>(a, s);
    default: return a.p.bf16 ? attn_launch<4, true>(a, s) : attn_launch<4, false>(a, s);
  }
}

}  // namespace mf
