// Rotary positions (gfx950): pairs of channels of queries and keys turned by their token's position.
#include <type_traits>

#include "mf_device.h"
#include "paged8.h"
#include "paged_attn.h"

namespace mf {

// ------------------------------------------------------------------------------------------
// k_rope: four tokens of some heads a workgroup. A wave computes the cosines and sines of one token into LDS, then a thread
// turns 16-byte pieces of rows (one and its partner rot / 2 channels on, or one whose pairs lie inside it). Where pairs do
// not lie in pieces like that (rot / 2 no multiple of 8, rot of interleaved pairs none), the rows go through LDS.
//
// The angle is p * r in 64 bits, reduced to a part of a turn there: in 32 bits position 10^6 would be off by up to 0.06 radians.
//
// y = m (u cos - v sin, v cos + u sin) of a pair (u, v): 4 bytes a channel read and written for two fused operations, so memory bounds
// it. A token's angles serve all of the workgroup's heads, whose first pieces of rows are under way while they are computed: 9600 tokens
// of 40 heads of 128, 198 MB, take 37 us, 5.3 TB/s. Through LDS only what is turned goes, and what is not is copied at once: 20 of 80
// channels of 4096 tokens of 64 heads, 84 MB, take 22 us, 3.8 TB/s (all channels through LDS, loaded behind the angles, 30 a call for 24.7);
// its two barriers and the conflicts of 2-byte reads, 40% of LDS's time, are the rest. 64 tokens take 3.7 us: a chain of latencies
// (start, length, angle, store).
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

template <int FORM, bool BF16, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void k_rope(RopeArgs a, int heads, int head_groups) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int valid[kRopeTokens];
  const bool half = a.layout == MUSTAFAR_ROPE_HALF;
  const int pairs = a.rot / 2, pad = (pairs + 7) & ~7, all = a.Hq + a.H;
  float* const turns = reinterpret_cast<float*>(smem);  // [kRopeTokens][cosines, sines][pad]
  // kRopeAny: [kRopeTokens][channels], and the rows' channels that are turned, up to a whole piece
  const int channels = (a.rot + 7) & ~7;
  float2* const factors = reinterpret_cast<float2*>(smem);
  uint16_t* const stage = reinterpret_cast<uint16_t*>(factors + kRopeTokens * channels);
  const int tile = (int)(blockIdx.x / head_groups), h0 = (int)(blockIdx.x % head_groups) * heads, nh = min(heads, all - h0);
  const int t0 = tile * kRopeTokens, wave = (int)(threadIdx.x / kWave), lane = (int)lane_id();
  // Row r of the workgroup: token r / nh, head h0 + r % nh. A thread has one piece of every step-th row.
  const bool in_place = (a.Hq == 0 || a.out_q == a.q) && (a.H == 0 || a.out_k == a.k);
  const int turned = FORM == kRopeHalf ? a.rot / 16 : (a.rot + 7) / 8;  // pieces that are turned; the others are copied
  const int pieces = in_place ? turned : FORM == kRopeAny ? a.d / 8 : turned + (a.d - a.rot) / 8;
  const int piece = (int)threadIdx.x % pieces, sub = (int)threadIdx.x / pieces, step = kRopeThreads / pieces;
  const int rows = sub < step ? kRopeTokens * nh : 0;
  const bool copied = piece >= turned;
  const int at = FORM == kRopeAny || !copied ? 8 * piece : a.rot + 8 * (piece - turned);
  auto from = [&](int tok, int h) {
    return h < a.Hq ? a.q + (int64_t)(t0 + tok) * a.q_stride + h * a.d : a.k + (int64_t)(t0 + tok) * a.k_stride + (h - a.Hq) * a.d;
  };
  auto to = [&](int tok, int h) {
    return h < a.Hq ? a.out_q + (int64_t)(t0 + tok) * a.out_q_stride + h * a.d
                    : a.out_k + (int64_t)(t0 + tok) * a.out_k_stride + (h - a.Hq) * a.d;
  };
  struct Item {
    u32x4 x, partner;
  };
  constexpr int kItems = FORM == kRopeAny ? 2 : 1;
  Item items[kItems];
  auto load = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int r = r0 + i * step, tok = r / nh;
      if (r >= rows || t0 + tok >= a.n) continue;
      const uint16_t* const x = from(tok, h0 + r - tok * nh) + at;
      const auto *const from_x = reinterpret_cast<const u32x4*>(x), *const from_z = reinterpret_cast<const u32x4*>(x + pairs);
      items[i].x = STREAM ? __builtin_nontemporal_load(from_x) : *from_x;
      if (FORM == kRopeHalf && !copied) items[i].partner = STREAM ? __builtin_nontemporal_load(from_z) : *from_z;
    }
  };
  load(sub);  // (under way while the angles are computed)
  {
    const RopeRow row = rope_row(a, t0 + wave);
    if (lane == 0) valid[wave] = row.valid;
    for (int i = lane; i < pairs; i += kWave) {
      double x = (double)row.pos * a.rates[i] * 0.15915494309189533577;  // of a turn
      x -= rint(x);
      float s, c;
      sincospif((float)(2 * x), &s, &c);
      c *= a.magnitude;
      s *= a.inverse ? -a.magnitude : a.magnitude;
      if constexpr (FORM == kRopeAny) {  // of each channel: what it and its partner are multiplied by
        factors[wave * channels + (half ? i : 2 * i)] = make_float2(c, -s);
        factors[wave * channels + (half ? i + pairs : 2 * i + 1)] = make_float2(c, s);
      } else {
        turns[(2 * wave) * pad + i] = c;
        turns[(2 * wave + 1) * pad + i] = s;
      }
    }
  }
  __syncthreads();
  for (int r0 = sub; r0 < rows; r0 += kItems * step) {
    if (r0 != sub) load(r0);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int r = r0 + i * step, tok = r / nh;
      if (r >= rows || !valid[tok]) continue;
      uint16_t* const y = to(tok, h0 + r - tok * nh) + at;
      const u32x4 x = items[i].x;
      if (copied) {
        *reinterpret_cast<u32x4*>(y) = x;
      } else if constexpr (FORM == kRopeAny) {
        *reinterpret_cast<u32x4*>(stage + r * channels + at) = x;
      } else if constexpr (FORM == kRopeHalf) {
        const u32x4 z = items[i].partner;
        const float *cosine = turns + 2 * tok * pad + at, *sine = cosine + pad;
        u32x4 ya, yb;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float p[2], q[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float u = to_float<BF16>(k ? x[e] >> 16 : x[e] & 0xffffu), v = to_float<BF16>(k ? z[e] >> 16 : z[e] & 0xffffu);
            const float c = cosine[2 * e + k], s = sine[2 * e + k];
            p[k] = fmaf(u, c, -v * s);
            q[k] = fmaf(v, c, u * s);
          }
          ya[e] = pack2<BF16>(p[0], p[1]);
          yb[e] = pack2<BF16>(q[0], q[1]);
        }
        *reinterpret_cast<u32x4*>(y) = ya;
        *reinterpret_cast<u32x4*>(y + pairs) = yb;
      } else {
        const float *cosine = turns + 2 * tok * pad + 4 * piece, *sine = cosine + pad;
        u32x4 ys;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = to_float<BF16>(x[e] & 0xffffu), v = to_float<BF16>(x[e] >> 16), c = cosine[e], s = sine[e];
          ys[e] = pack2<BF16>(fmaf(u, c, -v * s), fmaf(v, c, u * s));
        }
        *reinterpret_cast<u32x4*>(y) = ys;
      }
    }
  }
  if constexpr (FORM == kRopeAny) {
    __syncthreads();
    for (int i = (int)threadIdx.x; i < kRopeTokens * nh * turned; i += kRopeThreads) {
      const int r = i / turned, c8 = 8 * (i - r * turned), tok = r / nh;
      if (!valid[tok]) continue;
      const uint16_t* const x = stage + r * channels;
      const float2* const f = factors + tok * channels;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = c8 + e, other = half ? (c < pairs ? c + pairs : c - pairs) : c ^ 1;
        y[e] = to_float<BF16>(x[c]);
        if (c < a.rot) y[e] = fmaf(y[e], f[c].x, to_float<BF16>(x[other]) * f[c].y);
      }
      *reinterpret_cast<u32x4*>(to(tok, h0 + r - tok * nh) + c8) =
          (u32x4){pack2<BF16>(y[0], y[1]), pack2<BF16>(y[2], y[3]), pack2<BF16>(y[4], y[5]), pack2<BF16>(y[6], y[7])};
    }
  }
}

hipError_t launch_rope(const RopeArgs& a, const RopePlan& plan, hipStream_t s) {
  const size_t channels = (a.rot + 7) & ~7;
  const size_t lds = kRopeTokens * (plan.form == kRopeAny ? (8 + 2 * (size_t)plan.heads) * channels : 8 * (size_t)((a.rot / 2 + 7) & ~7));
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)plan.groups), dim3(kRopeThreads), lds, s, a, plan.heads, plan.head_groups);
  };
  // (a rotation that the last cache does not hold: 39.2 us for 41.6, 9600 tokens of 40 heads of 128, 198 MB read and written, whose
  // outputs stay there so; one of 84 MB that it holds takes 25.5 for 23.6)
  auto of_type = [&](auto form, auto stream) {
    constexpr int FORM = decltype(form)::value;
    constexpr bool STREAM = decltype(stream)::value;
    a.bf16 ? launch(k_rope<FORM, true, STREAM>) : launch(k_rope<FORM, false, STREAM>);
  };
  auto of_size = [&](auto form) {
    4 * (int64_t)a.n * (a.Hq + a.H) * a.d > kLastLevel / 2 ? of_type(form, std::true_type()) : of_type(form, std::false_type());
  };
  switch (plan.form) {
    case kRopeHalf: of_size(std::integral_constant<int, kRopeHalf>()); break;
    case kRopePairs: of_size(std::integral_constant<int, kRopePairs>()); break;
    default: of_size(std::integral_constant<int, kRopeAny>()); break;
  }
  return hipGetLastError();
}

}  // namespace mf
