// The paged dense cache (gfx950): a step's tables and slots from the requests'
// lengths, new keys and values into their slots, requests' pages as dense tensors.
#include "paged.h"

#include "mf_device.h"

namespace mf {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------
// k_paged_plan: lengths -> pages, tables, sequence starts, slots.
//
// With ob = ceil(len / P) pages held and nb = ceil(len' / P) needed, three prefix sums
// over the entries (new tokens, pages taken, pages given up) place everything else: the
// page given up as r-th lies at (the entry whose prefix holds r, nb + the rest) of the
// table, and the stack with them pushed on, last first, has the page taken as i-th at
// rank i from its top, so it is the page given up as i-th, or entry n_free - 1 - (i - R)
// of the old stack. Every workgroup computes the sums for itself (at most 4096 entries,
// in LDS) and does its share of the slots, taken and returned pages with binary
// searches; none waits for another: the table's entries that are written, [ob, nb), are
// those that nobody reads, and the stack is written only above its old top.
// In place, the lengths may be overwritten once every workgroup is done with them: the
// last one to take a ticket (the state's last word, back at 0 afterwards) writes them.
// A chain of memory latencies bounds it (lengths, prefix sums, table or stack, slot), so a thread has one slot until 65536:
// 64 requests of a token each take 4.2 us, 256 with up to 512 tokens (256 workgroups) 9.3; with four slots a thread 13.1.
// ------------------------------------------------------------------------------------------
constexpr int kPlanThreads = 256;
constexpr int kPlanPerGroup = 256;  // slots a workgroup
enum { kPlanPages = 1, kPlanTable = 2, kPlanSlots = 4, kPlanState = 8 };

struct PlanArgs {
  const int32_t* state;
  const int32_t* keep;
  const int32_t* new_len;
  int32_t* state_out;
  int32_t* table;
  int32_t* free_pages;
  int32_t* cu;
  int32_t* slots;
  int32_t* status;
  int B, log2_page, n_pages, max_pages, n_slots;
};

struct PlanEntry {
  int len, kept, add, ob, nb;
};

__device__ __forceinline__ PlanEntry plan_entry(const PlanArgs& a, int b) {
  PlanEntry e;
  e.len = a.state[b];
  e.kept = a.keep ? min(max(a.keep[b], 0), e.len) : e.len;
  e.add = a.new_len[b];
  const int up = (1 << a.log2_page) - 1;
  e.ob = (int)(((int64_t)e.len + up) >> a.log2_page);
  e.nb = (int)(((int64_t)e.kept + e.add + up) >> a.log2_page);
  return e;
}

// What is wrong with an entry; its counts are inside [0, MUSTAFAR_PAGED_MAX_STEP] when nothing
// is, so that 4096 of them add up inside 32 bits.
__device__ __forceinline__ int plan_wrong(const PlanArgs& a, const PlanEntry& e) {
  int w = 0;
  if (e.len < 0 || e.ob > a.max_pages || e.add < 0) w |= kPlanState;
  else if (e.nb > a.max_pages) w |= kPlanTable;
  if (e.add > a.n_slots) w |= kPlanSlots;
  return w;
}

// The entry whose range of the prefix sums at[0 .. B] holds i: the last b with at[b] <= i.
__device__ __forceinline__ int plan_find(const uint32_t* at, int B, uint32_t i) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kPlanThreads) void k_paged_plan(PlanArgs a) {
  extern __shared__ uint32_t sm[];  // cu, taken, given: [B + 1] each
  __shared__ uint32_t wsum[4][kPlanThreads / kWave];
  __shared__ int wbits[kPlanThreads / kWave];
  __shared__ int last;
  uint32_t* cu = sm;
  uint32_t* taken = sm + a.B + 1;
  uint32_t* given = sm + 2 * (a.B + 1);
  const int t = threadIdx.x, wave = t / kWave;
  const int per = (a.B + kPlanThreads - 1) / kPlanThreads;
  const int n_free = a.state[a.B];

  uint32_t sum[4] = {0u, 0u, 0u, 0u};  // new tokens, pages taken, given up, held
  int wrong = n_free < 0 || n_free > a.n_pages ? kPlanState : 0;
  for (int b = t * per; b < min(a.B, (t + 1) * per); ++b) {
    const PlanEntry e = plan_entry(a, b);
    const int w = plan_wrong(a, e);
    wrong |= w;
    if (!(w & kPlanState)) sum[3] += (uint32_t)e.ob;
    if (w) continue;
    sum[0] += (uint32_t)e.add;
    sum[1] += (uint32_t)max(e.nb - e.ob, 0);
    sum[2] += (uint32_t)max(e.ob - e.nb, 0);
  }
  uint32_t base[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t incl = wave_incl_scan(sum[k]);
    if (t % kWave == kWave - 1) wsum[k][wave] = incl;
    base[k] = incl - sum[k];
  }
  int bits = 0;
#pragma unroll
  for (int bit = 1; bit <= kPlanState; bit *= 2)
    if (ballot((wrong & bit) != 0)) bits |= bit;
  if (t % kWave == 0) wbits[wave] = bits;
  __syncthreads();
  uint32_t total[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    bits |= wbits[w];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (w < wave) base[k] += wsum[k][w];
      total[k] += wsum[k][w];
    }
  }
  // (no page is held twice, so that the pages given up have room on the stack)
  if ((int64_t)total[3] + n_free > a.n_pages) bits |= kPlanState;
  if (!bits) {
    if (total[0] > (uint32_t)a.n_slots) bits |= kPlanSlots;
    if (total[1] > total[2] && total[1] - total[2] > (uint32_t)n_free) bits |= kPlanPages;
  }
  const bool planned = bits == 0;
  for (int b = t * per; b < min(a.B, (t + 1) * per); ++b) {
    const PlanEntry e = plan_entry(a, b);
    cu[b] = planned ? base[0] : 0u;
    taken[b] = base[1];
    given[b] = base[2];
    base[0] += (uint32_t)e.add;
    base[1] += (uint32_t)max(e.nb - e.ob, 0);
    base[2] += (uint32_t)max(e.ob - e.nb, 0);
  }
  if (t == 0) {
    cu[a.B] = planned ? total[0] : 0u;
    taken[a.B] = total[1];
    given[a.B] = total[2];
  }
  __syncthreads();
  const uint32_t n_taken = planned ? total[1] : 0u, n_given = planned ? total[2] : 0u, n_new = planned ? total[0] : 0u;

  auto page_given = [&](uint32_t r) {
    const int b = plan_find(given, a.B, r);
    return a.table[(int64_t)b * a.max_pages + plan_entry(a, b).nb + (int)(r - given[b])];
  };
  auto page_taken = [&](uint32_t i) { return i < n_given ? page_given(i) : a.free_pages[n_free - 1 - (int)(i - n_given)]; };

  const uint32_t step = gridDim.x * kPlanThreads, first = blockIdx.x * kPlanThreads + t;
  for (uint32_t i = first; i < (uint32_t)a.n_slots; i += step) {
    int slot = -1;
    if (i < n_new) {
      const int b = plan_find(cu, a.B, i);
      const PlanEntry e = plan_entry(a, b);
      const int pos = e.kept + (int)(i - cu[b]), blk = pos >> a.log2_page;
      const int page = blk < e.ob ? a.table[(int64_t)b * a.max_pages + blk] : page_taken(taken[b] + (uint32_t)(blk - e.ob));
      slot = (page << a.log2_page) + (pos & ((1 << a.log2_page) - 1));
    }
    a.slots[i] = slot;
  }
  for (uint32_t i = first; i < n_taken; i += step) {
    const int b = plan_find(taken, a.B, i);
    a.table[(int64_t)b * a.max_pages + plan_entry(a, b).ob + (int)(i - taken[b])] = page_taken(i);
  }
  for (uint32_t r = n_taken + first; r < n_given; r += step) a.free_pages[n_free + (int)(n_given - 1 - r)] = page_given(r);

  if (blockIdx.x == 0) {
    for (int b = t; b <= a.B; b += kPlanThreads) a.cu[b] = (int)cu[b];
    if (t == 0) a.status[0] = bits;
  }
  // The new state: by the first workgroup, or in place by the last one that needed the old.
  if (a.state_out != a.state) {
    if (blockIdx.x != 0) return;
  } else if (gridDim.x > 1) {
    __syncthreads();
    if (t == 0)
      last = __hip_atomic_fetch_add(a.state_out + a.B + 1, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
  } else {
    __syncthreads();
  }
  for (int b = t; b < a.B; b += kPlanThreads) {
    const PlanEntry e = plan_entry(a, b);
    a.state_out[b] = planned ? e.kept + e.add : e.len;
  }
  if (t == 0) {
    a.state_out[a.B] = n_free + (int)n_given - (int)n_taken;
    a.state_out[a.B + 1] = 0;
  }
}

hipError_t launch_paged_plan(const PagedView& p, const int32_t* keep, const int32_t* new_len, int32_t* state_out,
                             int32_t* cu, int32_t* slots, int n_slots, int32_t* status, hipStream_t s) {
  const PlanArgs a = {p.state, keep, new_len, state_out, p.table, p.free_pages, cu, slots,
                      status,  p.B,  p.log2_page, p.n_pages, p.max_pages, n_slots};
  const int groups = n_slots > kPlanPerGroup ? (n_slots + kPlanPerGroup - 1) / kPlanPerGroup : 1;
  hipLaunchKernelGGL(k_paged_plan, dim3(groups < 256 ? groups : 256), dim3(kPlanThreads),
                     3 * sizeof(uint32_t) * (p.B + 1), s, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// k_paged_write: 16 bytes of a token's key and of its value a thread. Memory bounds it: 16384 tokens of 8 heads at d = 128 take
// 24 us (5.6 TB/s, reads and writes). Non-temporal stores take 22, but the attention that reads the pages next then
// takes 3 more.
// ------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_paged_write(PagedView p, const uint16_t* k_new, int64_t k_stride,
                                                    const uint16_t* v_new, int64_t v_stride, const int32_t* slots,
                                                    int64_t n_vec) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_vec) return;
  const int dv = p.d / 8, row = p.H * dv;
  const int64_t tok = i / row;
  const int c = (int)(i - tok * row), h = c / dv;
  const int slot = slots[tok], page = slot >> p.log2_page;
  if (slot < 0 || page >= p.n_pages) return;
  const int64_t dst = (int64_t)page * p.page_stride + (int64_t)h * p.head_stride +
                      (int64_t)(slot & ((1 << p.log2_page) - 1)) * p.token_stride + 8 * (c - h * dv);
  *reinterpret_cast<u32x4*>(p.k + dst) = *reinterpret_cast<const u32x4*>(k_new + tok * k_stride + 8 * c);
  *reinterpret_cast<u32x4*>(p.v + dst) = *reinterpret_cast<const u32x4*>(v_new + tok * v_stride + 8 * c);
}

hipError_t launch_paged_write(const PagedView& p, const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new,
                              int64_t v_stride, const int32_t* slots, int n_new, hipStream_t s) {
  // (a launch has less than 2^32 threads)
  const int64_t row = p.H * (p.d / 8), most = (((int64_t)1 << 32) - 512) / row;
  for (int64_t t = 0; t < n_new; t += most) {
    const int64_t n_vec = (n_new - t < most ? n_new - t : most) * row;
    hipLaunchKernelGGL(k_paged_write, dim3((uint32_t)((n_vec + 255) / 256)), dim3(256), 0, s, p, k_new + t * k_stride, k_stride,
                       v_new + t * v_stride, v_stride, slots + t, n_vec);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------------------------
// k_paged_gather: 16 bytes of a key row and of its value row a thread, a head's rows a run of workgroups. Memory bounds it:
// outputs of 537 MB take 112 us non-temporal (5.9 TB/s, reads and writes) and 132 through the caches (with a kernel that
// reads them next, 494 and 502); of 134 MB, which the last cache holds for that kernel, 128 and 117 with it.
// ------------------------------------------------------------------------------------------
constexpr int64_t kLastLevel = 256 << 20;  // bytes of the last cache

__device__ __forceinline__ uint32_t bf16_pair_to_fp16(uint32_t w) {
  uint32_t r = 0u;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float x = __builtin_bit_cast(float, i ? w & 0xffff0000u : w << 16);
    x = x > 65504.f ? 65504.f : x < -65504.f ? -65504.f : x;  // (NaN stays)
    r |= (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x) << (16 * i);
  }
  return r;
}

template <bool BF16, bool STREAM>
__global__ __launch_bounds__(256) void k_paged_gather(PagedView p, const int32_t* first, uint16_t* x_k, uint16_t* x_v,
                                                     int n_max, uint32_t groups) {
  const uint32_t bh = blockIdx.x / groups, b = bh / p.H, h = bh - b * p.H, log2_dv = 31 - __builtin_clz(p.d / 8);
  const int64_t i = (int64_t)(blockIdx.x - bh * groups) * 256 + threadIdx.x, j = i >> log2_dv;  // of the rows of b and h
  const int64_t tok = j + (first ? max(first[b], 0) : 0);
  if (j >= n_max || tok >= p.state[b] || tok >> p.log2_page >= p.max_pages) return;
  int page = p.table[(int64_t)b * p.max_pages + (tok >> p.log2_page)];
  if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
  const int64_t src = (int64_t)page * p.page_stride + (int64_t)h * p.head_stride +
                      (int64_t)(tok & ((1 << p.log2_page) - 1)) * p.token_stride + 8 * (i & ((1 << log2_dv) - 1));
  const int64_t dst = (int64_t)bh * n_max * p.d + 8 * i;
  const auto *from_k = reinterpret_cast<const u32x4*>(p.k + src), *from_v = reinterpret_cast<const u32x4*>(p.v + src);
  u32x4 k = STREAM ? __builtin_nontemporal_load(from_k) : *from_k, v = STREAM ? __builtin_nontemporal_load(from_v) : *from_v;
  if constexpr (BF16) {
    k = (u32x4){bf16_pair_to_fp16(k.x), bf16_pair_to_fp16(k.y), bf16_pair_to_fp16(k.z), bf16_pair_to_fp16(k.w)};
    v = (u32x4){bf16_pair_to_fp16(v.x), bf16_pair_to_fp16(v.y), bf16_pair_to_fp16(v.z), bf16_pair_to_fp16(v.w)};
  }
  auto *to_k = reinterpret_cast<u32x4*>(x_k + dst), *to_v = reinterpret_cast<u32x4*>(x_v + dst);
  if constexpr (STREAM) {
    __builtin_nontemporal_store(k, to_k);
    __builtin_nontemporal_store(v, to_v);
  } else {
    *to_k = k;
    *to_v = v;
  }
}

hipError_t launch_paged_gather(const PagedView& p, const int32_t* first, uint16_t* x_k, uint16_t* x_v, int n_max,
                               hipStream_t s) {
  const int64_t groups = ((int64_t)n_max * (p.d / 8) + 255) / 256, bh = (int64_t)p.B * p.H;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(bh * groups)), dim3(256), 0, s, p, first, x_k, x_v, n_max, (uint32_t)groups);
  };
  if (4 * bh * n_max * p.d > kLastLevel) p.bf16 ? launch(k_paged_gather<true, true>) : launch(k_paged_gather<false, true>);
  else p.bf16 ? launch(k_paged_gather<true, false>) : launch(k_paged_gather<false, false>);
  return hipGetLastError();
}

}  // namespace mf
