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
  const int64_t n_few = paged_parts(a.few_rows, a.few);
  float* const o = (float*)a.ws;
  const PartOut few = {(float2*)(o + n_few * (64 * T)), o, a.few_rows, a.by_entry, a.few};
  const int64_t tiles = paged_tiles(a.p, a.G, a.n_q, kFewRows);
  hipLaunchKernelGGL((k_paged8_rows<T, BF16, INT8>), dim3((uint32_t)(tiles * a.p.H * a.few)), dim3(kWave), 0, s, a, few);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_paged_merge(a, few, true, s);
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
