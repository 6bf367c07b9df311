// The paged cache in 8 bits (gfx950): a step's keys and values quantised into pages, requests' pages as
// dense tensors.
#include "codes.h"
#include "paged8.h"

namespace mf {

// ------------------------------------------------------------------------------------------
// k_paged8_write: a wave has 16 tokens of one head's keys or values, the waves of a block of tokens share a workgroup and
// their largest magnitude. The new tokens are read once and stay in registers; the block's earlier codes are read only where the
// new tokens raise its exponent. A workgroup's block is found from the starts and lengths, so that no two have the same one
// whatever the step.
//
// 2 bytes read and 1 written a channel, so memory bounds it: 16100 rows of 8 kv-heads of 128 in bf16, 99 MB, take 21.5 us, 4.6 TB/s.
// Keys and values of a head in one wave took 31.6 us for 27.8 (then); the new rows, which nothing reads again, past the caches made 41
// of 47 us for a write with its reading back. Single tokens of 64 requests take 4.2 us: starts and lengths, page, scale and codes in turn.
// ------------------------------------------------------------------------------------------
struct BlockTile {
  int b, row0, first, last;  // request, the row of its first new token, the positions of its first and last
  int block;                 // first position of the block (over `last`: nothing to do)
};

// New tokens of an entry: positions first .. last (last < first: none), of which `first` is row row0.
__device__ __forceinline__ BlockTile new_tokens(const PagedView& p, int b, int cu, int next, int len, int n_new) {
  BlockTile t;
  const int n = min(next, n_new) - cu;
  const int64_t most = (int64_t)p.max_pages << p.log2_page;
  t.b = b;
  t.last = (int)min((int64_t)max(len, 0), most) - 1;
  t.first = max(t.last + 1 - max(n, 0), 0);
  if (cu < 0) t.last = t.first - 1;
  t.row0 = cu + n - (t.last + 1 - t.first);
  t.block = 0;
  return t;
}

// Tile `tile` of the launch. n rows are in n / T + 2 blocks of T tokens at most, so that a request's tiles begin at cu / T + 2 b and
// the next one's behind them; a step of 4096 requests finds them as fast as one of 65.
__device__ __forceinline__ BlockTile block_tile(const PagedView& p, const int32_t* cu, int n_new, int log2_block, int tile) {
  auto start = [&](int c, int b) { return (c >> log2_block) + 2 * b; };
  const Request r = last_request(cu, p.state, p.B, [&](int c, int b) { return start(c, b) <= tile; });
  BlockTile t = new_tokens(p, r.b, r.cu, r.next, r.len, n_new);
  const int64_t block = ((int64_t)(t.first >> log2_block) + (tile - start(r.cu, r.b))) << log2_block;
  if (t.last < t.first || block > t.last) return {0, 0, 0, -1, 0};
  t.block = (int)block;
  return t;
}

template <int T, bool BF16, bool INT8>
__global__ __launch_bounds__(kWrite8Threads) void k_paged8_write(Paged8View c, const uint16_t* k_new, int64_t k_stride,
                                                                 const uint16_t* v_new, int64_t v_stride, const int32_t* cu,
                                                                 int n_new, int groups) {
  constexpr int kWaves = kWrite8Threads / kWave, kPieces = 8 * T, kRowsPerLoad = kWave / kPieces, kLoads = kWrite8Rows / kRowsPerLoad;
  __shared__ float tops[kWaves];
  const PagedView& p = c.p;
  const int tile = (int)(blockIdx.x / groups), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = (int)lane_id();
  const int log2_waves = c.log2_block - 4;  // of a head's block
  const int head = (int)(blockIdx.x % groups) * (kWaves >> log2_waves) + (wave >> log2_waves), sub = wave & ((1 << log2_waves) - 1);
  const BlockTile t = block_tile(p, cu, n_new, c.log2_block, tile);
  if (t.block > t.last) return;  // (all of the workgroup)
  const bool work = head < 2 * p.H, values = head >= p.H;
  const int h = work ? values ? head - p.H : head : 0, place = t.block & ((1 << p.log2_page) - 1);
  const uint16_t* const x_new = (values ? v_new : k_new) + h * p.d;
  const int64_t x_stride = values ? v_stride : k_stride;
  // Rows of this wave: positions t.block + row + kRowsPerLoad i. The new ones are under way while the page is looked up.
  const int row = kWrite8Rows * sub + lane / kPieces, c8 = 8 * (lane % kPieces);
  u32x4 x[kLoads];
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int pos = t.block + row + kRowsPerLoad * i, r = t.row0 + pos - t.first;
    x[i] = (u32x4){};
    if (work && pos >= t.first && pos <= t.last && r < n_new) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x_new + r * x_stride + c8));
  }
  const int page = p.table[(int64_t)t.b * p.max_pages + (t.block >> p.log2_page)];
  if ((uint32_t)page >= (uint32_t)p.n_pages) return;
  uint8_t* const codes = reinterpret_cast<uint8_t*>(values ? p.v : p.k) + (int64_t)page * p.page_stride + (int64_t)h * p.head_stride;
  uint8_t* const scale = (values ? c.v_scale : c.k_scale) + (((int64_t)page * p.H + h) << (p.log2_page - c.log2_block)) + (place >> c.log2_block);
  const bool older = t.block < t.first;
  const uint32_t before = older && work ? *scale : 0u;
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      top = fmaxf(top, fmaxf(fabsf(to_float<BF16>(x[i][e] & 0xffffu)), fabsf(to_float<BF16>(x[i][e] >> 16))));  // (not NaN's)
  top = wave_max(top);
  if (log2_waves > 0) {
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    for (int i = 0; i < 1 << log2_waves; ++i) top = fmaxf(top, tops[(wave & ~((1 << log2_waves) - 1)) + i]);
  }
  if (!work) return;
  const uint32_t byte = max(byte_for<BF16, INT8>(top), before);
  if (older && byte != before) {
    // 2^(before - byte), or, where that is no normal number, so little that every code becomes 0.
    const float less = power_of((uint32_t)max((int)before - (int)byte + 127, 1));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = row + kRowsPerLoad * i;
      if (t.block + r >= t.first) continue;
      u32x2* const at = reinterpret_cast<u32x2*>(codes + (int64_t)(place + r) * p.token_stride + c8);
      u32x2 y = *at;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const f32x4 f = decode4<INT8>(y[e], less);
        y[e] = encode4<INT8>(f[0], f[1], f[2], f[3]);
      }
      *at = y;
    }
  }
  const float inverse = power_of(254u - byte);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = row + kRowsPerLoad * i, pos = t.block + r;
    if (pos < t.first || pos > t.last) continue;
    *reinterpret_cast<u32x2*>(codes + (int64_t)(place + r) * p.token_stride + c8) =
        (u32x2){encode_pairs<BF16, INT8>(x[i][0], x[i][1], inverse), encode_pairs<BF16, INT8>(x[i][2], x[i][3], inverse)};
  }
  if (lane == 0 && sub == 0) *scale = (uint8_t)byte;
}

template <int T>
static hipError_t write8_launch(const Paged8View& c, const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new,
                                int64_t v_stride, const int32_t* cu, int n_new, hipStream_t s) {
  const int groups = paged8_block_groups(c.p, c.log2_block);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(paged8_blocks(c.p, c.log2_block, n_new) * groups)), dim3(kWrite8Threads), 0, s, c, k_new,
                       k_stride, v_new, v_stride, cu, n_new, groups);
  };
  if (c.int8) c.p.bf16 ? launch(k_paged8_write<T, true, true>) : launch(k_paged8_write<T, false, true>);
  else c.p.bf16 ? launch(k_paged8_write<T, true, false>) : launch(k_paged8_write<T, false, false>);
  return hipGetLastError();
}

hipError_t launch_paged8_write(const Paged8View& c, const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new,
                               int64_t v_stride, const int32_t* cu, int n_new, hipStream_t s) {
  switch (c.p.d) {
    case 64: return write8_launch<1>(c, k_new, k_stride, v_new, v_stride, cu, n_new, s);
    case 128: return write8_launch<2>(c, k_new, k_stride, v_new, v_stride, cu, n_new, s);
    default: return write8_launch<4>(c, k_new, k_stride, v_new, v_stride, cu, n_new, s);
  }
}

// ------------------------------------------------------------------------------------------
// k_paged8_gather: 8 codes of a key row and of its value row a thread, a head's rows a run of workgroups.
//
// 1 byte read and 2 written a channel, so memory bounds it: 166 + 331 MB take 85 to 92 us, 5.4 to 5.8 TB/s, past the last cache, which cannot hold
// them for their reader (through it 100 us); 25 MB, which it holds, 6.3 us, 3.9 TB/s with the launch's start and end.
// ------------------------------------------------------------------------------------------
template <bool INT8>
__device__ __forceinline__ u32x2 codes_to_fp16(uint32_t codes, float scale) {
  f32x4 x = decode4<INT8>(codes, scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = x[i] > 65504.f ? 65504.f : x[i] < -65504.f ? -65504.f : x[i];  // (NaN stays)
  return (u32x2){pack2<false>(x[0], x[1]), pack2<false>(x[2], x[3])};
}

template <bool INT8, bool STREAM>
__global__ __launch_bounds__(256) void k_paged8_gather(Paged8View c, const int32_t* first, uint16_t* x_k, uint16_t* x_v,
                                                      int n_max, uint32_t groups) {
  const PagedView& p = c.p;
  const uint32_t bh = blockIdx.x / groups, b = bh / p.H, h = bh - b * p.H, log2_dv = 31 - __builtin_clz(p.d / 8);
  const int64_t i = (int64_t)(blockIdx.x - bh * groups) * 256 + threadIdx.x, j = i >> log2_dv;  // of the rows of b and h
  const int64_t tok = j + (first ? max(first[b], 0) : 0);
  if (j >= n_max || tok >= p.state[b] || tok >> p.log2_page >= p.max_pages) return;
  int page = p.table[(int64_t)b * p.max_pages + (tok >> p.log2_page)];
  if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
  const int place = (int)(tok & ((1 << p.log2_page) - 1));
  const int64_t src = (int64_t)page * p.page_stride + (int64_t)h * p.head_stride + (int64_t)place * p.token_stride + 8 * (i & ((1 << log2_dv) - 1));
  const int64_t block = (((int64_t)page * p.H + h) << (p.log2_page - c.log2_block)) + (place >> c.log2_block);
  const int64_t dst = (int64_t)bh * n_max * p.d + 8 * i;
  const auto* const from_k = reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(p.k) + src);
  const auto* const from_v = reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(p.v) + src);
  const u32x2 k = STREAM ? __builtin_nontemporal_load(from_k) : *from_k, v = STREAM ? __builtin_nontemporal_load(from_v) : *from_v;
  const float ks = power_of(c.k_scale[block]), vs = power_of(c.v_scale[block]);
  const u32x2 k0 = codes_to_fp16<INT8>(k.x, ks), k1 = codes_to_fp16<INT8>(k.y, ks);
  const u32x2 v0 = codes_to_fp16<INT8>(v.x, vs), v1 = codes_to_fp16<INT8>(v.y, vs);
  const u32x4 dense_k = {k0.x, k0.y, k1.x, k1.y}, dense_v = {v0.x, v0.y, v1.x, v1.y};
  auto *const to_k = reinterpret_cast<u32x4*>(x_k + dst), *const to_v = reinterpret_cast<u32x4*>(x_v + dst);
  if constexpr (STREAM) {
    __builtin_nontemporal_store(dense_k, to_k);
    __builtin_nontemporal_store(dense_v, to_v);
  } else {
    *to_k = dense_k;
    *to_v = dense_v;
  }
}

hipError_t launch_paged8_gather(const Paged8View& c, const int32_t* first, uint16_t* x_k, uint16_t* x_v, int n_max,
                                hipStream_t s) {
  const int64_t groups = ((int64_t)n_max * (c.p.d / 8) + 255) / 256, bh = (int64_t)c.p.B * c.p.H;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(bh * groups)), dim3(256), 0, s, c, first, x_k, x_v, n_max, (uint32_t)groups);
  };
  if (4 * bh * n_max * c.p.d > kLastLevel) c.int8 ? launch(k_paged8_gather<true, true>) : launch(k_paged8_gather<false, true>);
  else c.int8 ? launch(k_paged8_gather<true, false>) : launch(k_paged8_gather<false, false>);
  return hipGetLastError();
}

}  // namespace mf
