// Causal attention of the new tokens of every request over its pages (gfx950), with an
// optional sliding window and first tokens that stay visible.
#include "mf_device.h"
#include "paged.h"

namespace mf {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <bool BF16>
__device__ __forceinline__ float to_float(uint32_t bits) {
  if constexpr (BF16) return __builtin_bit_cast(float, bits << 16);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

template <bool BF16>
__device__ __forceinline__ uint16_t from_float(float x) {
  if constexpr (BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
  else return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// The request of row t: the last b with cu[b] <= t.
__device__ __forceinline__ int request_of(const int32_t* cu, int B, int t) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Element offset of token j of entry b, kv-head h.
__device__ __forceinline__ int64_t token_at(const PagedView& p, int b, int h, int j) {
  int page = p.table[(int64_t)b * p.max_pages + (j >> p.log2_page)];
  if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
  return (int64_t)page * p.page_stride + (int64_t)h * p.head_stride +
         (int64_t)(j & ((1 << p.log2_page) - 1)) * p.token_stride;
}

// The least weight of a visible token: an infinite value that one sees stays infinite
// where its probability is under fp32's range (0 times infinity would be NaN).
constexpr float kLeast = 0x1p-120f;
__device__ __forceinline__ float at_least(float x) { return x < kLeast ? kLeast : x; }  // (NaN stays)

// One wave per row and query head, 64 tokens at a time: lane = token for the scores, lane =
// channel for the values.
template <int T, bool BF16>
__global__ __launch_bounds__(64) void k_paged_attn_row(PagedAttnArgs a) {
  constexpr int d = kTile * T;
  __shared__ float qs[d];
  const PagedView& p = a.p;
  const int t = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, h = hq / a.G;
  if (t >= a.cu[p.B]) return;
  const uint32_t lane = lane_id();
  const int b = request_of(a.cu, p.B, t);
  const int64_t most = (int64_t)p.max_pages << p.log2_page;
  const int len = (int)min((int64_t)max(p.state[b], 0), most);
  const int pos = len - (a.cu[b + 1] - t);
#pragma unroll
  for (int c = 0; c < T; ++c) qs[lane + kTile * c] = to_float<BF16>(a.q[t * a.q_stride + hq * d + kTile * c + lane]);
  __syncthreads();
  const int lo = a.window > 0 ? max(pos - a.window + 1, 0) : 0, sinks = min(a.sinks, lo);
  const int n = pos < 0 ? 0 : sinks + pos + 1 - lo;
  float m = -INFINITY, l = 0.f, o[T];
#pragma unroll
  for (int c = 0; c < T; ++c) o[c] = 0.f;
  for (int u0 = 0; u0 < n; u0 += kWave) {
    const int u = min(u0 + (int)lane, n - 1);
    const int64_t at = token_at(p, b, h, u < sinks ? u : lo + u - sinks);
    float s = 0.f;
#pragma unroll 4
    for (int c = 0; c < d; c += 8) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p.k + at + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s = fmaf(qs[c + 2 * e], to_float<BF16>(w[e] & 0xffffu), s);
        s = fmaf(qs[c + 2 * e + 1], to_float<BF16>(w[e] >> 16), s);
      }
    }
    if (u0 + (int)lane >= n) s = -INFINITY;
    const float mnew = fmaxf(m, wave_max(s));
    const float alpha = m == -INFINITY ? 1.f : at_least(__builtin_amdgcn_exp2f((m - mnew) * a.scale_log2));
    float w = s == -INFINITY ? 0.f : at_least(__builtin_amdgcn_exp2f((s - mnew) * a.scale_log2));
    m = mnew;
    l = fmaf(l, alpha, wave_sum(w));
#pragma unroll
    for (int c = 0; c < T; ++c) o[c] *= alpha;
    for (int i = 0; i < min(kWave, n - u0); ++i) {
      const float wi = __shfl(w, i, kWave);
      const int64_t ai = __shfl(at, i, kWave);
#pragma unroll
      for (int c = 0; c < T; ++c) o[c] = fmaf(wi, to_float<BF16>(p.v[ai + kTile * c + lane]), o[c]);
    }
  }
#pragma unroll
  for (int c = 0; c < T; ++c)
    a.out[t * a.out_stride + hq * d + kTile * c + lane] = from_float<BF16>(n > 0 ? o[c] / l : 0.f);
}

template <int T>
static hipError_t attn_T(const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid((uint32_t)a.n_q * (uint32_t)a.Hq);
  if (a.p.bf16) hipLaunchKernelGGL((k_paged_attn_row<T, true>), grid, dim3(kWave), 0, s, a);
  else hipLaunchKernelGGL((k_paged_attn_row<T, false>), grid, dim3(kWave), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.p.d) {
    case 64: return attn_T<1>(a, s);
    case 128: return attn_T<2>(a, s);
    default: return attn_T<4>(a, s);
  }
}

}  // namespace mf
