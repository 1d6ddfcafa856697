// Pages, block tables and slots of a round (ts_kv_plan).
//
// The free pages are a stack.  A request's need is a division of its length;
// which stack entry each page goes to or comes from is a prefix sum over the
// requests, so one workgroup scans them and moves the pages.  Bound by launch and
// latency: a call for one request takes 2.8 us on the device, one for 256 requests
// (16400 pages taken) 12.4 us and 4 for the slots.
#pragma once

#include "kv_format.hpp"

namespace ts {

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
template <int THREADS>
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
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    const int x = lds[w];
    if (w < wave) before += x;
    total += x;
  }
  return v + before;
}

// The slot of row i of a request.
__device__ __forceinline__ int plan_slot(const KvPlanParams& p, const int32_t* row, int len, int granted, int i) {
  if (i > granted) return -1;
  const int pos = len + i;  // a granted request's positions fit its table
  const int page = kv_page(row, pos >> p.page_shift, p.max_blocks, p.num_pages);
  return page < 0 ? -1 : (page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
}

// One workgroup; requests in rounds of THREADS.  SLOTS: it writes the slot map
// too (small ones: the call is then a single launch).
template <int THREADS, bool SLOTS>
__global__ __launch_bounds__(THREADS) void kv_plan_kernel(KvPlanParams p) {
  __shared__ int sums[THREADS / 64], taken;
  __shared__ int first[THREADS], from[THREADS], upto[THREADS];
  const int t = threadIdx.x;
  const int count0 = min(max(*p.free_count, 0), p.num_pages);
  if (t == 0) taken = 0;
  // The pages that a round's requests give back or take, from number first[r]
  // below the stack's top on: a wave takes four requests at a time and sends the
  // loads of up to 128 pages of each before it writes any.
  auto move = [&](int q0, int top, bool give) {
    constexpr int kWaves = THREADS / 64;
    const int n = min(THREADS, p.R - q0), lane = t & 63;
    for (int r0 = t >> 6; r0 < n; r0 += 4 * kWaves) {
      int lo[4], hi[4], most = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int r = r0 + u * kWaves;
        lo[u] = r < n ? from[r] : 0, hi[u] = r < n ? upto[r] : 0;
        most = max(most, hi[u] - lo[u]);
      }
      for (int d = lane; d - lane < most; d += 128) {
        int value[4][2];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = r0 + u * kWaves, b = lo[u] + d + 64 * j;
            value[u][j] = -1;
            if (b < hi[u]) {
              const int slot = top - 1 - (first[r] + d + 64 * j);
              if (give) value[u][j] = p.table[(size_t)(q0 + r) * p.max_blocks + b];
              else if (slot < p.num_pages) value[u][j] = p.free_pages[slot];
            }
          }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = r0 + u * kWaves, b = lo[u] + d + 64 * j;
            if (b >= hi[u]) continue;
            const int slot = top - 1 - (first[r] + d + 64 * j);
            if (give && slot < p.num_pages) p.free_pages[slot] = value[u][j];
            p.table[(size_t)(q0 + r) * p.max_blocks + b] = give ? -1 : value[u][j];
          }
      }
    }
  };
  // pages given back; their total first where there are several rounds
  PlanNeed x = {0, 0, false};
  int total, back = 0, given = 0;
  if (p.R > THREADS)
    for (int q0 = 0; q0 < p.R; q0 += THREADS) {
      if (q0 + t < p.R) x = plan_need(p, q0 + t);
      plan_scan<THREADS>(q0 + t < p.R && x.fits ? max(x.held - x.need, 0) : 0, sums, total);
      back += total;
    }
  for (int q0 = 0; q0 < p.R; q0 += THREADS) {
    if (q0 + t < p.R) x = plan_need(p, q0 + t);
    const int v = q0 + t < p.R && x.fits ? max(x.held - x.need, 0) : 0;
    const int incl = plan_scan<THREADS>(v, sums, total);
    if (p.R <= THREADS) back = total;
    if (back == 0) break;
    first[t] = given + incl - v;
    from[t] = x.need;
    upto[t] = x.need + v;
    __syncthreads();
    move(q0, count0 + back, true);
    __syncthreads();
    given += total;
  }
  const int top = count0 + back;
  // pages taken: each request whole or not at all
  int lack = 0;
  for (int q0 = 0; q0 < p.R; q0 += THREADS) {
    const int q = q0 + t;
    if (p.R > THREADS && q < p.R) x = plan_need(p, q);
    const int v = q < p.R && x.fits ? max(x.need - x.held, 0) : 0;
    const int incl = lack + plan_scan<THREADS>(v, sums, total);
    const bool ok = x.fits && (v == 0 || incl <= top);
    if (q < p.R) {
      const int nodes = min(p.n[q], p.cap - 1);
      if (ok) p.held[q] = x.need;
      p.granted[q] = ok && nodes >= 0 ? nodes : -1;
    }
    if (total == 0) continue;  // nothing lacks here
    // sums only grow, so the largest that is served is the sum of what is
    if (ok && v) atomicMax(&taken, incl);
    first[t] = incl - v;
    from[t] = x.held;
    upto[t] = ok ? x.held + v : x.held;
    __syncthreads();
    move(q0, top, false);
    __syncthreads();
    lack += total;
  }
  __syncthreads();
  if (t == 0) *p.free_count = min(top - taken, p.num_pages);
  if constexpr (SLOTS) {
    // what the workgroup wrote to the tables and to `granted` is there: its barriers
    // order it, and all of it went through one compute unit
    for (int s = t; s < p.R * p.cap; s += THREADS) {
      const int q = s / p.cap;
      p.slot[s] = plan_slot(p, p.table + (size_t)q * p.max_blocks, max(p.len[q], 0), p.granted[q], s - q * p.cap);
    }
  }
}

constexpr int kSlotThreads = 256;
__global__ __launch_bounds__(kSlotThreads) void kv_slot_kernel(KvPlanParams p) {
  const int q = blockIdx.x;
  const int len = max(p.len[q], 0), granted = p.granted[q];
  const int32_t* row = p.table + (size_t)q * p.max_blocks;
  int32_t* out = p.slot + (size_t)q * p.cap;
  for (int i = blockIdx.y * kSlotThreads + threadIdx.x; i < p.cap; i += gridDim.y * kSlotThreads)
    out[i] = plan_slot(p, row, len, granted, i);
}

}  // namespace ts
