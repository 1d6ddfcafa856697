// Attention over the 4-bit cache under the tree mask (ts_kv_attention).
//
// out = sum_t w_t V_t / sum_t w_t with w_t = exp(scale <Q, K_t> - max), in one
// pass over the tokens with a running maximum.
#pragma once

#include "kv_format.hpp"

namespace ts {

__device__ __forceinline__ float kv_load(const float* x) { return *x; }
__device__ __forceinline__ float kv_load(const __bf16* x) { return (float)*x; }
__device__ __forceinline__ void kv_store(float* x, float v) { *x = v; }
__device__ __forceinline__ void kv_store(__bf16* x, float v) { *x = (__bf16)v; }

// A wave per (request, row, query head): 64 tokens at a time, first a lane to
// a token for the scores, then a lane to D / 64 elements for the sums.
constexpr int kAttnWaves = 4;
template <typename TE, int D>
__global__ __launch_bounds__(64 * kAttnWaves) void kv_attention_kernel(KvAttnParams p) {
  __shared__ float q_lds[kAttnWaves][D], w_lds[kAttnWaves][64];
  __shared__ int page_lds[kAttnWaves][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * kAttnWaves + wave;
  if (item >= (int64_t)p.R * p.cap * p.q_heads) return;
  const int a = (int)(item % p.q_heads), i = (int)(item / p.q_heads % p.cap), q = (int)(item / p.q_heads / p.cap);
  const int shift = p.c.page_shift, limit = p.max_blocks << shift;
  const KvRows x = kv_rows(p.len, p.n, q, p.cap, limit);
  if (i >= x.rows) return;
  const int head = a / p.group;
  const int32_t* table = p.table + (size_t)q * p.max_blocks;
  const TE* qr = static_cast<const TE*>(p.q) + ((int64_t)q * p.cap + i) * p.q_stride + a * D;
  for (int d = lane; d < D; d += 64) q_lds[wave][d] = kv_load(qr + d);
  wave_lds_sync();
  const uint32_t* bits = p.mask ? p.mask + ((size_t)q * p.cap + i) * p.mask_words : nullptr;
  const int total = x.len + (bits ? x.rows : i + 1);
  float m = kNegInf, l = 0.f, o[D / 64];
  for (float& v : o) v = 0.f;
  for (int t0 = 0; t0 < total; t0 += 64) {
    const int t = t0 + lane, j = t - x.len;
    const bool sees = t < total && (j < 0 || !bits || (bits[j >> 5] >> (j & 31) & 1u));
    const int page = sees ? kv_page(table, t >> shift, p.max_blocks, p.c.num_pages) : -1;
    const int off = t & ((1 << shift) - 1);
    float s = kNegInf;
    if (sees) {
      s = __builtin_nanf("");
      if (page >= 0) {
        const char* b = kv_block<D>(p.c, page, head);
        s = 0.f;
        for (int g = 0; g < D / 32; ++g) {
          const uint32_t sc = (uint8_t)b[KvBlock<D>::key_scales(off, shift) + g];
          float dot = 0.f;
          for (int w = 0; w < 4; ++w) {
            const uint32_t codes = *reinterpret_cast<const uint32_t*>(b + KvBlock<D>::key_codes(off) + g * 16 + w * 4);
            bf16x2 k[4];
            fp4_to_bf16x8(codes, sc == 255 ? 127u : sc, k);
            for (int e = 0; e < 4; ++e) {
              dot = __builtin_fmaf(q_lds[wave][g * 32 + w * 8 + 2 * e], (float)k[e][0], dot);
              dot = __builtin_fmaf(q_lds[wave][g * 32 + w * 8 + 2 * e + 1], (float)k[e][1], dot);
            }
          }
          s += sc == 255 ? __builtin_nanf("") : dot;
        }
        s *= p.scale_log2;
      }
    }
    const float top = fmaxf(m, wave_max(s));
    const float at = top == kNegInf ? 0.f : top;
    const float w = sees ? exp2_fast(s - at) : 0.f, keep = exp2_fast(m - at);
    l = l * keep + wave_sum(w);
    m = top;
    w_lds[wave][lane] = w;
    page_lds[wave][lane] = page;
    wave_lds_sync();
    for (float& v : o) v *= keep;
    for (int u = 0; u < min(64, total - t0); ++u) {
      const int pg = page_lds[wave][u], of = (t0 + u) & ((1 << shift) - 1);
      if (pg < 0) continue;
      const char* b = kv_block<D>(p.c, pg, head);
      const float wu = w_lds[wave][u];
      for (int e = 0; e < D / 64; ++e) {
        const int d = lane + 64 * e;
        const uint32_t sc = (uint8_t)b[KvBlock<D>::value_scales(of, shift) + d / 32];
        const uint32_t code = (uint8_t)b[KvBlock<D>::value_codes(of, shift) + d / 2];
        bf16x2 v[4];
        fp4_to_bf16x8(sc == 255 ? 0u : code, value_scale(sc), v);
        o[e] = __builtin_fmaf(wu, (float)v[0][d & 1], o[e]);
      }
    }
    wave_lds_sync();
  }
  TE* out = static_cast<TE*>(p.out) + (((int64_t)q * p.cap + i) * p.q_heads + a) * D;
  for (int e = 0; e < D / 64; ++e) kv_store(out + lane + 64 * e, l == 0.f ? 0.f : o[e] / l);
  if (p.lse && lane == 0)
    p.lse[((int64_t)q * p.cap + i) * p.q_heads + a] = l == 0.f ? kNegInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace ts
