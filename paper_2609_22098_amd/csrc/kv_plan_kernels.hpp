// Pages, block tables and slots of a round (ts_kv_plan).
//
// The free pages are a stack.  A request's need is a division of its length;
// which stack entry each page goes to or comes from is a prefix sum over the
// requests, so one workgroup scans them.  The stack entries that one request
// moves are consecutive: a wave moves them together.
#pragma once

#include "kv_format.hpp"

namespace ts {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// What a request has and needs.
struct PlanNeed {
  int held, need;  // pages
  bool fits;       // in the table
};
__device__ __forceinline__ PlanNeed plan_need(const KvPlanParams& p, int q) {
  const int nodes = min(p.n[q], p.cap - 1);
  const int64_t want = (int64_t)max(p.len[q], 0) + max(nodes + 1, 0);
  const int64_t need = (want + (1 << p.page_shift) - 1) >> p.page_shift;
  return {min(max(p.held[q], 0), p.max_blocks), (int)min(need, (int64_t)p.max_blocks), need <= p.max_blocks};
}

// Inclusive sum over the workgroup's threads, and the total in `total`.
__device__ __forceinline__ int plan_scan(int v, int* lds, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(v, d);
    if (lane >= d) v += x;
  }
  __syncthreads();  // the previous scan's sums have been read
  if (lane == 63) lds[wave] = v;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < kPlanWaves; ++w) {
    const int x = lds[w];
    if (w < wave) before += x;
    total += x;
  }
  return v + before;
}

__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(KvPlanParams p) {
  __shared__ int sums[kPlanWaves];
  __shared__ int first[kPlanThreads], from[kPlanThreads], upto[kPlanThreads];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int count0 = min(max(*p.free_count, 0), p.num_pages);
  // pages given back
  int total, back = 0;
  for (int q0 = 0; q0 < p.R; q0 += kPlanThreads) {
    int v = 0;
    if (q0 + t < p.R) {
      const PlanNeed x = plan_need(p, q0 + t);
      v = x.fits ? max(x.held - x.need, 0) : 0;
    }
    plan_scan(v, sums, total);
    back += total;
  }
  const int top = count0 + back;
  int base = 0;
  for (int q0 = 0; q0 < p.R && back > 0; q0 += kPlanThreads) {
    PlanNeed x = {0, 0, false};
    if (q0 + t < p.R) x = plan_need(p, q0 + t);
    const int v = x.fits ? max(x.held - x.need, 0) : 0;
    const int incl = plan_scan(v, sums, total);
    first[t] = base + incl - v;
    from[t] = x.need;
    upto[t] = x.need + v;
    __syncthreads();
    for (int r = wave; r < kPlanThreads && q0 + r < p.R; r += kPlanWaves) {
      int32_t* row = p.table + (size_t)(q0 + r) * p.max_blocks;
      for (int b = from[r] + lane; b < upto[r]; b += 64) {
        const int at = top - 1 - (first[r] + b - from[r]);
        if (at < p.num_pages) p.free_pages[at] = row[b];
        row[b] = -1;
      }
    }
    __syncthreads();
    base += total;
  }
  // pages taken: each request whole or not at all
  int lack = 0, taken = 0;
  for (int q0 = 0; q0 < p.R; q0 += kPlanThreads) {
    const int q = q0 + t;
    PlanNeed x = {0, 0, false};
    if (q < p.R) x = plan_need(p, q);
    const int v = x.fits ? max(x.need - x.held, 0) : 0;
    const int incl = lack + plan_scan(v, sums, total);
    const bool ok = x.fits && (v == 0 || incl <= top);
    first[t] = incl - v;
    from[t] = x.held;
    upto[t] = ok ? x.held + v : x.held;
    lack += total;
    plan_scan(ok ? v : 0, sums, total);  // its barriers also publish the arrays above
    taken += total;
    for (int r = wave; r < kPlanThreads && q0 + r < p.R; r += kPlanWaves) {
      int32_t* row = p.table + (size_t)(q0 + r) * p.max_blocks;
      for (int b = from[r] + lane; b < upto[r]; b += 64) {
        const int at = top - 1 - (first[r] + b - from[r]);
        row[b] = at < p.num_pages ? p.free_pages[at] : -1;
      }
    }
    __syncthreads();  // every wave has read the arrays and p.held
    if (q < p.R) {
      const int nodes = min(p.n[q], p.cap - 1);
      if (ok) p.held[q] = x.need;
      p.granted[q] = ok && nodes >= 0 ? nodes : -1;
    }
  }
  if (t == 0) *p.free_count = min(top - taken, p.num_pages);
}

// Slots of the granted rows, four a thread.
constexpr int kSlotThreads = 256;
__global__ __launch_bounds__(kSlotThreads) void kv_slot_kernel(KvPlanParams p) {
  const int q = blockIdx.x;
  const int len = max(p.len[q], 0), granted = p.granted[q];
  const int32_t* row = p.table + (size_t)q * p.max_blocks;
  int32_t* out = p.slot + (size_t)q * p.cap;
  const int mask = (1 << p.page_shift) - 1;
  for (int i = blockIdx.y * kSlotThreads + threadIdx.x; i < p.cap; i += gridDim.y * kSlotThreads) {
    int slot = -1;
    if (i <= granted) {
      const int pos = len + i;  // a granted request's positions fit its table
      const int page = kv_page(row, pos >> p.page_shift, p.max_blocks, p.num_pages);
      if (page >= 0) slot = (page << p.page_shift) + (pos & mask);
    }
    out[i] = slot;
  }
}

}  // namespace ts
