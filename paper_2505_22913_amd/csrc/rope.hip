// Rotary positions (gfx950): pairs of channels of queries and keys turned by their token's position.
#include <type_traits>

#include "mf_device.h"
#include "paged8.h"
#include "paged_attn.h"

namespace mf {

// ------------------------------------------------------------------------------------------
// k_rope: four tokens of some heads a workgroup. A wave computes the cosines and sines of one token into LDS, then a thread
// turns 16-byte pieces of rows: one and its partner rot / 2 channels on (W = 8), or one whose pairs lie in it (W = 0). Where rot / 2 is no
// multiple of 8, the pieces go through LDS, where a thread turns W channels and their partners.
//
// The angle is p * r in 64 bits, reduced to a part of a turn there: in 32 bits position 10^6 would be off by up to 0.06 radians.
//
// y = m (u cos - v sin, v cos + u sin) of a pair (u, v): 4 bytes a channel read and written for two fused operations, so memory bounds
// it. A token's angles serve all of the workgroup's heads, whose first pieces are under way while they are computed: 9600 tokens of 40
// heads of 128, 198 MB, take 35 us (38 one launch behind the other), 5.6 TB/s, interleaved or in halves. Through LDS 20 of 80 channels of 4096 tokens of 64 heads, 84 MB, take 18 to 23 us, 3.6 to 4.7 TB/s:
// the rest of a row is copied past it, and the pairs are turned where they lie (each piece gathering its partners by itself there took
// 24.6, without LDS by loads and stores of W channels 57: their number). Divisions are products with inverses from the host: 38.3 us for 40.5 and
// 3.1 for 3.3 with 64 tokens, which are a chain of latencies (start, length, angle, store).
// ------------------------------------------------------------------------------------------
// What a row's request is, of row t of a step.
struct RopeRow {
  int64_t pos;
  bool valid;
};
__device__ __forceinline__ RopeRow rope_row(const RopeArgs& a, int t) {
  if (a.positions) return {t < a.n ? (int64_t)a.positions[t] : 0, t < a.n};
  const Request r = request_at(a.cu, a.state, a.B, t);
  const int64_t len = min((int64_t)max(r.len, 0), a.most);
  return {len - min(r.next, a.n) + t, t < a.n && t < a.cu[a.B]};
}

// N floats of LDS (aligned as so many, or as four).
template <int N>
__device__ __forceinline__ void load_floats(const float* x, float (&y)[N]) {
  if constexpr (N < 4) {
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = x[e];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(x + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[i + e] = v[e];
    }
  }
}

// W channels (two bytes each, from the first word's lower half on) and their partners turned.
template <bool BF16, int W, int N>
__device__ __forceinline__ void turn(uint32_t (&x)[N], uint32_t (&z)[N], const float* cosine, const float* sine) {
  float c[W], s[W];
  load_floats(cosine, c);
  load_floats(sine, s);
#pragma unroll
  for (int e = 0; e < W; e += 2) {
    float p[2] = {}, q[2] = {};
#pragma unroll
    for (int k = 0; k < 2 && e + k < W; ++k) {
      const float u = to_float<BF16>(k ? x[e / 2] >> 16 : x[e / 2] & 0xffffu), v = to_float<BF16>(k ? z[e / 2] >> 16 : z[e / 2] & 0xffffu);
      p[k] = fmaf(u, c[e + k], -v * s[e + k]);
      q[k] = fmaf(v, c[e + k], u * s[e + k]);
    }
    x[e / 2] = pack2<BF16>(p[0], p[1]);
    z[e / 2] = pack2<BF16>(q[0], q[1]);
  }
}

template <int W, bool BF16, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void k_rope(RopeArgs a, RopePlan plan) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int valid[kRopeTokens];
  constexpr bool kLds = W != 0 && W != 8;
  const int pairs = a.rot / 2, pad = (pairs + 7) & ~7, whole = (a.rot + 7) & ~7;
  float* const turns = reinterpret_cast<float*>(smem);  // [kRopeTokens][cosines, sines][pad]
  uint16_t* const stage = reinterpret_cast<uint16_t*>(turns + 2 * kRopeTokens * pad);  // kLds: [rows][whole]
  const int tile = (int)((uint64_t)blockIdx.x * plan.groups_inverse >> 40);
  const int h0 = (int)(blockIdx.x - (uint32_t)tile * (uint32_t)plan.head_groups) * plan.heads, nh = min(plan.heads, a.Hq + a.H - h0);
  const int t0 = tile * kRopeTokens, wave = (int)(threadIdx.x / kWave), lane = (int)lane_id();
  const int rows = kRopeTokens * nh, items = rows * plan.pieces;
  auto token_of = [&](int r) { return (r >= nh) + (r >= 2 * nh) + (r >= 3 * nh); };
  auto from = [&](int tok, int h) {
    const int64_t t = t0 + tok;
    return h < a.Hq ? a.q + t * a.q_stride + h * a.d : a.k + t * a.k_stride + (h - a.Hq) * a.d;
  };
  auto to = [&](int tok, int h) {
    const int64_t t = t0 + tok;
    return h < a.Hq ? a.out_q + t * a.out_q_stride + h * a.d : a.out_k + t * a.out_k_stride + (h - a.Hq) * a.d;
  };
  // Item i: a piece of row i / pieces, whose rows are each token's heads.
  struct Item {
    int r, tok, h, at;
    bool turned;
  };
  auto item = [&](int i) __attribute__((always_inline)) {
    Item m;
    m.r = (int)((uint32_t)i * plan.pieces_inverse >> 24);
    const int piece = i - m.r * plan.pieces;
    m.tok = token_of(m.r);
    m.h = h0 + m.r - m.tok * nh;
    m.turned = piece < plan.turned;
    m.at = 8 * piece + (W == 8 && !m.turned ? pairs : 0);
    return m;
  };
  u32x4 x = {}, partner = {};
  auto load = [&](const Item& m) __attribute__((always_inline)) {
    if (t0 + m.tok >= a.n) return;
    const uint16_t* const y = from(m.tok, m.h) + m.at;
    const auto *const from_x = reinterpret_cast<const u32x4*>(y), *const from_z = reinterpret_cast<const u32x4*>(y + pairs);
    x = STREAM ? __builtin_nontemporal_load(from_x) : *from_x;
    if (W == 8 && m.turned) partner = STREAM ? __builtin_nontemporal_load(from_z) : *from_z;
  };
  Item m = item((int)threadIdx.x);
  if ((int)threadIdx.x < items) load(m);  // (under way while the angles are computed)
  {
    const RopeRow row = rope_row(a, t0 + wave);
    if (lane == 0) valid[wave] = row.valid;
    for (int i = lane; i < pairs; i += kWave) {
      double x = (double)row.pos * a.rates[i] * 0.15915494309189533577;  // of a turn
      x -= rint(x);
      float s, c;
      sincospif((float)(2 * x), &s, &c);
      turns[(2 * wave) * pad + i] = c * a.magnitude;
      turns[(2 * wave + 1) * pad + i] = s * (a.inverse ? -a.magnitude : a.magnitude);
    }
  }
  __syncthreads();
  for (int i = (int)threadIdx.x; i < items; i += kRopeThreads) {
    if (i != (int)threadIdx.x) {
      m = item(i);
      load(m);
    }
    if (!valid[m.tok]) continue;
    uint16_t* const y = to(m.tok, m.h) + m.at;
    const float* const cosine = turns + 2 * m.tok * pad;
    if (kLds && m.turned) {
      *reinterpret_cast<u32x4*>(stage + m.r * whole + m.at) = x;
      continue;
    }
    if (m.turned) {
      uint32_t u[4] = {x[0], x[1], x[2], x[3]};
      if constexpr (W == 8) {
        uint32_t v[4] = {partner[0], partner[1], partner[2], partner[3]};
        turn<BF16, 8>(u, v, cosine + m.at, cosine + pad + m.at);
        *reinterpret_cast<u32x4*>(y + pairs) = (u32x4){v[0], v[1], v[2], v[3]};
      } else {
        float c[4], s[4];
        load_floats(cosine + m.at / 2, c);
        load_floats(cosine + pad + m.at / 2, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = to_float<BF16>(x[e] & 0xffffu), q = to_float<BF16>(x[e] >> 16);
          if (m.at + 2 * e < a.rot) u[e] = pack2<BF16>(fmaf(p, c[e], -q * s[e]), fmaf(q, c[e], p * s[e]));
        }
      }
      x = (u32x4){u[0], u[1], u[2], u[3]};
    }
    *reinterpret_cast<u32x4*>(y) = x;
  }
  if constexpr (kLds) {
    typedef std::conditional_t<W == 4, u32x2, std::conditional_t<W == 2, uint32_t, uint16_t>> Channels;
    __syncthreads();
    for (int i = (int)threadIdx.x; i < rows * plan.units; i += kRopeThreads) {
      const int r = (int)((uint32_t)i * plan.units_inverse >> 24), at = W * (i - r * plan.units);
      const float* const cosine = turns + 2 * token_of(r) * pad + at;
      Channels *const x = reinterpret_cast<Channels*>(stage + r * whole + at), *const z = reinterpret_cast<Channels*>(stage + r * whole + at + pairs);
      uint32_t u[(W + 1) / 2], v[(W + 1) / 2];
      if constexpr (W == 4) {
        u[0] = x->x, u[1] = x->y, v[0] = z->x, v[1] = z->y;
        turn<BF16, W>(u, v, cosine, cosine + pad);
        *x = (u32x2){u[0], u[1]};
        *z = (u32x2){v[0], v[1]};
      } else {
        u[0] = *x, v[0] = *z;
        turn<BF16, W>(u, v, cosine, cosine + pad);
        *x = (Channels)u[0];
        *z = (Channels)v[0];
      }
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < rows * plan.turned; i += kRopeThreads) {
      const int r = i / plan.turned, at = 8 * (i - r * plan.turned), tok = token_of(r);
      if (valid[tok]) *reinterpret_cast<u32x4*>(to(tok, h0 + r - tok * nh) + at) = *reinterpret_cast<const u32x4*>(stage + r * whole + at);
    }
  }
}

hipError_t launch_rope(const RopeArgs& a, const RopePlan& plan, hipStream_t s) {
  const size_t turns = kRopeTokens * 8 * (size_t)((a.rot / 2 + 7) & ~7);
  const size_t lds = turns + (plan.width == 0 || plan.width == 8 ? 0 : kRopeTokens * 2 * (size_t)plan.heads * ((a.rot + 7) & ~7));
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)plan.groups), dim3(kRopeThreads), lds, s, a, plan);
  };
  // (a rotation that the last cache does not hold: 38.0 us for 39.6, 9600 tokens of 40 heads of 128, 198 MB read and written, whose
  // outputs stay there so; one of 84 MB that it holds takes 25.0 for 19.8 to 23.3)
  const bool stream = 4 * (int64_t)a.n * (a.Hq + a.H) * a.d > kLastLevel / 2;
  auto of_width = [&](auto width) {
    constexpr int W = decltype(width)::value;
    if (stream) a.bf16 ? launch(k_rope<W, true, true>) : launch(k_rope<W, false, true>);
    else a.bf16 ? launch(k_rope<W, true, false>) : launch(k_rope<W, false, false>);
  };
  switch (plan.width) {
    case 0: of_width(std::integral_constant<int, 0>()); break;
    case 8: of_width(std::integral_constant<int, 8>()); break;
    case 4: of_width(std::integral_constant<int, 4>()); break;
    case 2: of_width(std::integral_constant<int, 2>()); break;
    default: of_width(std::integral_constant<int, 1>()); break;
  }
  return hipGetLastError();
}

}  // namespace mf
