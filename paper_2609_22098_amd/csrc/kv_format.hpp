// The 4-bit key-value cache on the device: where a row lies and what its bytes mean.
//
// A block (layer, page, kv head) holds, for a page of P tokens and D values a
// head, key codes [P][D/2], key scales [P][D/32], value codes [P][D/2] and
// value scales [P][D/32].  A token's codes are contiguous, so that the 16 bytes
// a lane reads are 32 elements under one scale: the matrix unit's own fp4
// operand with its block scale.
#pragma once

#include "device_common.hpp"
#include "../../include/treespark_kv.h"

namespace ts {

struct KvView {
  char* pages;          // of the call's (first) layer
  int64_t layer_stride, page_stride;
  int num_pages, page_shift, heads;
};

// Byte offsets in a block of 2^page_shift tokens.
template <int D>
struct KvBlock {
  __device__ static int key_codes(int off) { return off * (D / 2); }
  __device__ static int key_scales(int off, int shift) { return (D / 2 << shift) + off * (D / 32); }
  __device__ static int value_codes(int off, int shift) { return ((D / 2 + D / 32) << shift) + off * (D / 2); }
  __device__ static int value_scales(int off, int shift) { return ((D + D / 32) << shift) + off * (D / 32); }
  __device__ static int bytes(int shift) { return (D * 17 / 16) << shift; }
};

// Block of a page for one head; page in [0, num_pages).
template <int D>
__device__ __forceinline__ char* kv_block(const KvView& c, int page, int head) {
  return c.pages + (int64_t)page * c.page_stride + (int64_t)head * KvBlock<D>::bytes(c.page_shift);
}

// Page of block b of a request's table row; -1 where there is none.
__device__ __forceinline__ int kv_page(const int32_t* table_row, int b, int max_blocks, int num_pages) {
  if (b >= max_blocks) return -1;
  const int page = table_row[b];
  return (uint32_t)page < (uint32_t)num_pages ? page : -1;
}

// Rows of request q: its context length and number of new rows.  A length past
// the table's last position is cut to one position past it: that one lies in no
// page, which is all that the longer context would say, and loops stay bounded.
struct KvRows {
  int len, rows;
};
__device__ __forceinline__ KvRows kv_rows(const int32_t* len, const int32_t* n, int q, int cap, int limit) {
  return {min(max(len[q], 0), limit + 1), max(min(n[q], cap - 1), -1) + 1};
}

// The eight values of a word of codes under a scale byte, as pairs of bf16
// (exact: a code has two significant bits).  The conversion takes the
// scale's exponent field.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void fp4_to_bf16x8(uint32_t codes, uint32_t scale_byte, bf16x2 (&out)[4]) {
  const float s = __uint_as_float(scale_byte << 23);
  out[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0);
  out[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1);
  out[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2);
  out[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3);
}

// A value's scale as attention reads it: 255 stands for zero values, and the
// clamp keeps every value finite (a masked one is multiplied by a weight of 0).
__device__ __forceinline__ uint32_t value_scale(uint32_t s) { return min(s, 252u); }

// Eight consecutive elements as fp32.
__device__ __forceinline__ void load8(const float* x, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(x), b = *reinterpret_cast<const f32x4*>(x + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[i + 4] = b[i];
}
__device__ __forceinline__ void load8(const __bf16* x, float (&v)[8]) {
  const u32x4 a = *reinterpret_cast<const u32x4*>(x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(a[i] << 16);
    v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
  }
}

// LDS written by lanes of a wave is read by others of the same wave: LDS works in
// program order there, so only the compiler has to keep the order.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Launch parameters -----------------------------------------------------
struct KvPlanParams {
  const int32_t *len, *n;
  int R, cap, page_shift, num_pages, max_blocks;
  int32_t *free_pages, *free_count, *held, *table, *slot, *granted;
};

struct KvAppendParams {
  KvView c;
  const void *k, *v;
  int64_t k_stride, v_stride;  // elements
  const int32_t* slot;
  int rows;
};

struct KvReadParams {
  KvView c;
  const int32_t* slot;
  int rows, layers;
  void *k, *v;
};

struct KvAcceptParams {
  KvView c;
  int layers;
  const int32_t *len, *n, *table, *path_nodes, *path_len;
  int R, max_blocks;
  int32_t* new_len;
};

// Row tiles of the attention kernel: rows of a workgroup's tile and its waves (see AttnShape).
enum class AttnTile : int { k16, k32, k64, k128 };

// A partial result's statistics: what weights are taken against (base-2 units),
// their sum, and the sum of what the products took of them.
struct alignas(16) AttnStat {
  float m, l, r, unused;
};
// A row tile whose parts a second kernel joins; q < 0: none.
struct AttnJoin {
  int q, head, m0, rows;
  int first;  // slot of its first part; the others are 2 w, 2 (w + 1), ...
  int last;   // workgroup of the last part
};

struct KvAttnParams {
  KvView c;
  const void* q;
  int64_t q_stride;  // elements
  int q_heads, group, R, cap, max_blocks, mask_words;
  const int32_t *len, *n, *table;
  const uint32_t* mask;
  float scale_log2;  // scale * log2(e): scores in base-2 units
  void* out;
  float* lse;
  int min_tokens;  // of a workgroup's piece
  int spare;       // workgroups left over for padding tiles to whole pieces; 0: no padding
  int whole_tiles; // tiles of a request and kv head, one a workgroup; 0: cut pieces
  float* parts;    // [2 * workgroups][rows of a tile][D]
  AttnStat* stats; // [2 * workgroups][rows of a tile]
  AttnJoin* joins; // [workgroups]
};

}  // namespace ts
