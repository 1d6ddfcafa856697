// Rows into the 4-bit cache, back out of it, and from place to place
// (ts_kv_append, ts_kv_read, ts_kv_accept).  Bound by bytes where there are many:
// 16384 rows of 8 heads of 128, 85 MB, take 20.6 us in and 18.9 us out (4.1 and 4.5
// TB/s; 16 and 16.6 us where the last-level cache still holds them); one request's
// take a launch, 2.8 us.
#pragma once

#include "kv_format.hpp"

namespace ts {

constexpr int kRowThreads = 256;

// Largest magnitude of a group's 32 elements, its four lanes (a quad) agreeing;
// the bits of magnitudes order as integers do, NaN and infinity on top.
__device__ __forceinline__ uint32_t group_max_bits(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  m = max(m, (uint32_t)dpp_i32<0xB1>((int)m));
  return max(m, (uint32_t)dpp_i32<0x4E>((int)m));
}

// The scale byte of a group: the least e with m <= 7 * 2^(e - 127).  The
// mantissa of 7 is 1.75: adding just less than what lies above it carries into
// the exponent exactly where m is more.  The lower bound keeps 127 - e a normal
// exponent, the upper one 6 * 2^(e - 127) finite.
__device__ __forceinline__ int group_scale(uint32_t max_bits) {
  return min(max((int)((max_bits + 0x1FFFFFu) >> 23) - 2, 2), 252);
}

// Codes of eight values: v_cvt rounds value / scale to the nearest E2M1, ties
// to the even code, and saturates at 6.
__device__ __forceinline__ uint32_t encode8(const float (&v)[8], int e) {
  const float s = __uint_as_float((uint32_t)e << 23);
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
}

// Eight elements of a key and of the value a thread: D / 8 neighbouring lanes
// hold a (row, head), four a group.
template <typename TE, int D>
__global__ __launch_bounds__(kRowThreads) void kv_append_kernel(KvAppendParams p) {
  constexpr int kLanes = D / 8;
  const int64_t item = (int64_t)blockIdx.x * (kRowThreads / kLanes) + threadIdx.x / kLanes;
  const int at = threadIdx.x % kLanes;
  const int row = (int)(item / p.c.heads), head = (int)(item % p.c.heads);
  if (row >= p.rows) return;
  const int slot = p.slot[row], shift = p.c.page_shift;
  if (slot < 0 || (slot >> shift) >= p.c.num_pages) return;
  float k[8], v[8];
  load8(static_cast<const TE*>(p.k) + (int64_t)row * p.k_stride + head * D + at * 8, k);
  load8(static_cast<const TE*>(p.v) + (int64_t)row * p.v_stride + head * D + at * 8, v);
  const uint32_t mk = group_max_bits(k), mv = group_max_bits(v);
  // a NaN or an infinity anywhere in the head
  uint32_t worst = max(mk, mv);
#pragma unroll
  for (int d = 4; d < kLanes; d <<= 1) worst = max(worst, (uint32_t)__shfl_xor((int)worst, d));
  const bool bad = worst >= 0x7F800000u;
  int ek = group_scale(mk), ev = group_scale(mv);
  const uint32_t ck = bad ? 0u : encode8(k, ek), cv = bad ? 0u : encode8(v, ev);
  if (bad) ek = 255, ev = 2;
  const int off = slot & ((1 << shift) - 1);
  char* b = kv_block<D>(p.c, slot >> shift, head);
  *reinterpret_cast<uint32_t*>(b + KvBlock<D>::key_codes(off) + at * 4) = ck;
  *reinterpret_cast<uint32_t*>(b + KvBlock<D>::value_codes(off, shift) + at * 4) = cv;
  if (at % 4 == 0) {
    b[KvBlock<D>::key_scales(off, shift) + at / 4] = (char)ek;
    b[KvBlock<D>::value_scales(off, shift) + at / 4] = (char)ev;
  }
}

// Eight elements a thread, key and value.
template <typename TE, int D>
__device__ __forceinline__ void store8(TE* out, uint32_t codes, uint32_t scale, bool zero, bool nan) {
  bf16x2 x[4];
  fp4_to_bf16x8(zero ? 0u : codes, zero || nan ? 127u : scale, x);
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = nan ? 0x7FC07FC0u : __builtin_bit_cast(uint32_t, x[i]);
  if constexpr (sizeof(TE) == 2) {
    *reinterpret_cast<u32x4*>(out) = w;
  } else {
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      a[2 * i] = __uint_as_float(w[i] << 16), a[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      b[2 * i] = __uint_as_float(w[i + 2] << 16), b[2 * i + 1] = __uint_as_float(w[i + 2] & 0xFFFF0000u);
    }
    *reinterpret_cast<f32x4*>(out) = a;
    *reinterpret_cast<f32x4*>(out + 4) = b;
  }
}

template <typename TE, int D>
__global__ __launch_bounds__(kRowThreads) void kv_read_kernel(KvReadParams p) {
  constexpr int kLanes = D / 8;
  const int64_t item = (int64_t)blockIdx.x * (kRowThreads / kLanes) + threadIdx.x / kLanes;
  const int at = threadIdx.x % kLanes, layer = blockIdx.y;
  const int row = (int)(item / p.c.heads), head = (int)(item % p.c.heads);
  if (row >= p.rows) return;
  const int slot = p.slot[row], shift = p.c.page_shift;
  if (slot < 0 || (slot >> shift) >= p.c.num_pages) return;
  const int off = slot & ((1 << shift) - 1);
  const char* b = kv_block<D>(p.c, slot >> shift, head) + layer * p.c.layer_stride;
  const int64_t to = (((int64_t)layer * p.rows + row) * p.c.heads + head) * D + at * 8;
  if (p.k) {
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(b + KvBlock<D>::key_codes(off) + at * 4);
    const uint32_t scale = (uint8_t)b[KvBlock<D>::key_scales(off, shift) + at / 4];
    store8<TE, D>(static_cast<TE*>(p.k) + to, codes, scale, false, scale == 255);
  }
  if (p.v) {
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(b + KvBlock<D>::value_codes(off, shift) + at * 4);
    const uint32_t scale = (uint8_t)b[KvBlock<D>::value_scales(off, shift) + at / 4];
    store8<TE, D>(static_cast<TE*>(p.v) + to, codes, scale, scale == 255, false);
  }
}

// The accepted rows of a request in one layer.  A thread owns a piece of the
// rows of one head (16 bytes of codes, or a row's scales), reads it of all accepted
// rows and then writes it, so that no order among the rows matters (a row's new
// place may be another's old one).  The path is looked up by a wave, a lane to a
// node.  Bound by lines of 128 bytes, of which a row's codes use 64 and its scales 4 (64
// requests, 32 layers, 8 heads: 30 us for 17 MB moved, 26 where the last-level cache
// still holds them); one request's 8.9 us are
// the path's, the table's and the rows' round trips.
template <int BYTES>
struct KvPiece;
template <>
struct KvPiece<2> { typedef uint16_t type; };
template <>
struct KvPiece<4> { typedef uint32_t type; };
template <>
struct KvPiece<8> { typedef uint64_t type; };
template <>
struct KvPiece<16> { typedef u32x4 type; };

// Moves a piece of BYTES at offset `at` + off * step of each row's block.
template <int BYTES, int D>
__device__ __forceinline__ void kv_move(char* base, const int64_t* src, const int64_t* dst, const int* src_off,
                                        const int* dst_off, int kept, int at, int step) {
  typedef typename KvPiece<BYTES>::type T;
  T w[TS_MAX_D];
#pragma unroll
  for (int j = 0; j < TS_MAX_D; ++j)
    if (j < kept) w[j] = *reinterpret_cast<const T*>(base + src[j] + at + src_off[j] * step);
#pragma unroll
  for (int j = 0; j < TS_MAX_D; ++j)
    if (j < kept) *reinterpret_cast<T*>(base + dst[j] + at + dst_off[j] * step) = w[j];
}

constexpr int kAcceptThreads = 128;
template <int D>
__global__ __launch_bounds__(kAcceptThreads) void kv_accept_kernel(KvAcceptParams p) {
  constexpr int kCodes = D / 32, kPieces = 2 * kCodes + 2;  // of a row of one head
  __shared__ int64_t src[TS_MAX_D], dst[TS_MAX_D];  // pages' first bytes
  __shared__ int src_off[TS_MAX_D], dst_off[TS_MAX_D], count;
  const int q = blockIdx.x, layer = blockIdx.y, t = threadIdx.x;
  const int shift = p.c.page_shift, limit = p.max_blocks << shift, mask = (1 << shift) - 1;
  if (t < 64) {
    const int n = p.n[q], paths = p.path_len[q], given = p.len[q], len = max(given, 0);
    const int node = t < TS_MAX_D ? p.path_nodes[q * TS_MAX_D + t] : 0;
    const int one_up = __shfl_up(node, 1), before = t ? one_up : 0;
    const bool on = n >= 0 && paths >= 0;
    bool valid = on && t < min(paths, TS_MAX_D) && len < limit && node > before && node <= n && node < limit - len;
    if (valid) {
      const int32_t* row = p.table + (size_t)q * p.max_blocks;
      const int a = len + node, b = len + 1 + t;  // b <= a: the path's nodes increase from 1 on
      const int pa = kv_page(row, a >> shift, p.max_blocks, p.c.num_pages);
      const int pb = b < limit ? kv_page(row, b >> shift, p.max_blocks, p.c.num_pages) : -1;
      valid = pa >= 0 && pb >= 0;
      if (valid) {
        src[t] = (int64_t)pa * p.c.page_stride, src_off[t] = a & mask;
        dst[t] = (int64_t)pb * p.c.page_stride, dst_off[t] = b & mask;
      }
    }
    const int kept = __builtin_ctzll(~__ballot(valid));  // up to the first that is not
    if (t == 0) {
      count = kept;
      if (layer == 0) p.new_len[q] = on ? len + 1 + kept : given;
    }
  }
  __syncthreads();
  const int kept = count;
  if (kept == 0) return;
  const int items = p.c.heads * kPieces;
  char* pages = p.c.pages + (int64_t)layer * p.c.layer_stride;
  for (int it = t; it < items; it += kAcceptThreads) {
    const int head = it / kPieces, piece = it % kPieces;
    char* base = pages + (int64_t)head * KvBlock<D>::bytes(shift);
    if (piece < kCodes)
      kv_move<16, D>(base, src, dst, src_off, dst_off, kept, KvBlock<D>::key_codes(0) + piece * 16, D / 2);
    else if (piece < 2 * kCodes)
      kv_move<16, D>(base, src, dst, src_off, dst_off, kept, KvBlock<D>::value_codes(0, shift) + (piece - kCodes) * 16, D / 2);
    else
      kv_move<D / 32, D>(base, src, dst, src_off, dst_off, kept,
                         piece == 2 * kCodes ? KvBlock<D>::key_scales(0, shift) : KvBlock<D>::value_scales(0, shift), D / 32);
  }
}

}  // namespace ts
