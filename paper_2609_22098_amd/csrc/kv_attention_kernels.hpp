// Attention over the 4-bit cache under the tree mask (ts_kv_attention).
//
// out = sum_t w_t V_t / sum_t w_t with w_t = exp(scale <Q, K_t> - max), in one
// pass over the tokens with a running maximum.
//
// Rows.  The query heads of a group share a kv head, so the rows of a product
// are (tree row, head of the group) pairs: row m = i * group + g of request q
// and kv head h.  A workgroup takes a tile of them.
//
// Scores.  S^T = K Q^T on the scaled matrix instruction 16x16x128: its A operand
// is the cache as it lies (16 tokens, 32 E2M1 codes and their scale byte a
// lane), so keys are never unpacked.  Its B operand has 8 bits: a query is cut
// into two E4M3 pieces of 4 significant bits, the second holding what the first
// left.  The instruction adds eight neighbouring products at a time and cuts them
// off, toward zero, below 2^(x - 13), x the largest sum of two operands'
// exponents.  So the first piece has no more bits than that: scaled by a power of
// two to at most 3.75, it has an exponent of at most 1 beside a key's 2, and its
// least step of 2^-9 (E4M3's) times a key's 1/2 is 2^(3 - 13): nothing is lost.
// (Scaled to [2, 4) what lies above 3.875 rounds up to 4, an exponent of 2: seven
// small products beside such a one were off by 3e-4 of it.)  What is smaller goes
// to the second piece, taken 2^8 times, whose step is then 2^-17.  It is at most
// 2^-4 of its element: of eight products, less than 7 * 2^-17 of the largest
// |Q| |K| is cut off.
// fp32 queries take three bf16 pieces and keys unpacked to bf16 (exact).
//
// Values.  O^T = V^T P^T on 16x16x32 bf16 (a value of the cache is exact in
// bf16).  Values are unpacked once per workgroup into LDS, [token][element],
// and read back transposed.  The scores' layout (a lane holds four consecutive
// tokens of one query) is the B operand's, so weights never leave their lane.
// An fp32 weight is cut into three bf16 pieces, a weight for bf16 outputs is
// rounded to one: its error is then as the output's own rounding.
//
// Work.  The steps of all tiles of all requests, in one line, are cut into
// equal pieces, one a workgroup: no length decides the balance.  A tile
// that a cut goes through leaves partial results, and a second kernel joins them.
// Where there are few tiles, each is padded to whole pieces; where a table names
// few tokens, nothing is cut: a workgroup takes a tile.
//
// Bounds.  Tiles of 16 rows: bytes (128 requests of one row over 300 to 16000
// tokens, 557 MB: 118 us, 4.7 TB/s; 131001 tokens of one: 32 us, 4.4 TB/s).  Tiles of
// 128: matrix and vector issue (prompts of 8000 rows over 2000 to 8000 tokens, 675
// GFLOP: 630 us, 1.07 PFLOP/s, and 21 for the join, once the clocks have risen: 710
// in the first twenty calls; 64 trees over 500 to 8000: 169 us and 18).  Few short
// contexts: round trips (a tree of 65 rows over 5003 tokens: 23 us and 7, of which 8
// are steps).
#pragma once

#include "kv_format.hpp"

namespace ts {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// A tile of 16 * MB * WM rows; WT waves take token tiles in turn, WM waves share
// one of them.  kRuns: pages that a token tile may touch: one where pages hold
// at least a tile (whose addresses are then one base and fixed steps), else four.
template <int D_, int MB_, int WM_, int WT_, typename TE_, bool WHOLE_>
struct AttnShape {
  static constexpr int D = D_, MB = MB_, WM = WM_, WT = WT_;
  using TE = TE_;
  static constexpr bool kF32 = sizeof(TE) == 4;
  static constexpr int kThreads = 64 * WM * WT;
  static constexpr int kTile = 64;               // tokens
  static constexpr int kRuns = WHOLE_ ? 1 : 4;
  static constexpr int kRows = 16 * MB * WM;     // of a workgroup's tile
  static constexpr int kQ = kF32 ? 3 : 2;        // pieces of a query
  static constexpr int kP = kF32 ? 3 : 1;        // pieces of a weight
  static constexpr int kKSteps = D <= 128 ? 1 : D / 128;
  static constexpr int kVRow = 2 * D + 32;       // bytes of a token in LDS: 4 rows of a transposed read on 32 banks
  static constexpr int kVTokens = WM == 1 ? 32 : 192;  // a wave's half tile; three whole tiles where waves share
  static constexpr int kORow = D + 4;            // floats of a row of results in LDS
  static constexpr int kVBytes = WT * kVTokens * kVRow;
  static constexpr int kOBytes = WT * WM * 16 * kORow * 4;
  static constexpr int kFixed = 512;             // tokens' worth of a tile's beginning and end (128: 64 trees 220 us, 128 single rows 147; this 190 and 124)
  // workgroups on a compute unit: registers allow waves of 128 where a wave has one block of rows
  static constexpr int kResident = MB == 1 && D <= 128 && !kF32 ? 3 : D <= 128 ? 2 : 1;
  static constexpr int kLds = kVBytes > kOBytes ? kVBytes : kOBytes;
};

// A wave's 16 queries as the score products' B operand (lane: query `col`, 32
// elements of each 128).
template <typename S, bool F32 = S::kF32>
struct AttnQuery;

template <typename S>
struct AttnQuery<S, false> {
  i32x8 w[S::kKSteps][2];
  int scales;  // of the pieces, a byte each: products come out as <Q, K> itself, whatever the query's size

  // The lane's elements as they are, and a step that uses them apart from it, so
  // that other loads can be sent in between.
  u32x4 raw[S::kKSteps][4];
  __device__ __forceinline__ void fetch(const __bf16* x, int quarter) {
#pragma unroll
    for (int k = 0; k < S::kKSteps; ++k)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int base = k * 128 + (u / 2) * 64;  // the instruction's order of 8-bit elements
        if (base < S::D) raw[k][u] = *reinterpret_cast<const u32x4*>(x + base + quarter * 16 + u % 2 * 8);
        else raw[k][u] = u32x4{0, 0, 0, 0};
      }
  }

  // sign: the scale's, 0 for none.
  __device__ __forceinline__ void convert(float sign) {
    float v[S::kKSteps][32];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < S::kKSteps; ++k)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[k][8 * u + 2 * j] = __uint_as_float(raw[k][u][j] << 16);
          v[k][8 * u + 2 * j + 1] = __uint_as_float(raw[k][u][j] & 0xFFFF0000u);
          top = max(top, raw[k][u][j] & 0x7FFF0000u);
          top = max(top, (raw[k][u][j] << 16) & 0x7FFF0000u);
        }
    top = max(top, (uint32_t)xor16_i32((int)top));
    top = max(top, (uint32_t)xor32_i32((int)top));
    // x * 2^(128 - e) has its largest in [1.9375, 3.875), which E4M3 rounds to at most 3.75 (below
    // 2^-118 it stays smaller, so that both scales are bytes: bf16's least is a whole step there)
    const int e = max((int)((top + 0x80000u) >> 23), 9);
    scales = (e - 1) | (e - 9) << 8;
    const bool finite = top < 0x7F800000u;  // else up is 0, and not-a-number comes of it
    const float up = sign * __uint_as_float(e < 255 ? (uint32_t)(255 - e) << 23 : finite ? 0x400000u : 0u);
#pragma unroll
    for (int k = 0; k < S::kKSteps; ++k)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = v[k][4 * u + j] * up;
        int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        word = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true);
        w[k][0][u] = word;
        y[0] = (y[0] - __builtin_amdgcn_cvt_f32_fp8(word, 0)) * 256.f;
        y[1] = (y[1] - __builtin_amdgcn_cvt_f32_fp8(word, 1)) * 256.f;
        y[2] = (y[2] - __builtin_amdgcn_cvt_f32_fp8(word, 2)) * 256.f;
        y[3] = (y[3] - __builtin_amdgcn_cvt_f32_fp8(word, 3)) * 256.f;
        word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        w[k][1][u] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true);
      }
  }

  // Product `i` of kProducts with 128 elements of 16 keys: small ones first.
  static constexpr int kProducts = 2;
  __device__ __forceinline__ f32x4 product(int i, i32x4 codes, int scale, int k, f32x4 acc) const {
    const i32x8 a = {codes[0], codes[1], codes[2], codes[3], 0, 0, 0, 0};
    return i == 0 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, w[k][1], acc, 4, 0, 0, scale, 1, scales)
                  : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, w[k][0], acc, 4, 0, 0, scale, 0, scales);
  }
};

template <typename S>
struct AttnQuery<S, true> {
  static constexpr float kBf16Max = 0x1.FEp127f;
  bf16x8 w[S::kKSteps][4][3];

  f32x4 raw[S::kKSteps][8];
  __device__ __forceinline__ void fetch(const float* x, int quarter) {
#pragma unroll
    for (int k = 0; k < S::kKSteps; ++k)
#pragma unroll
      for (int u = 0; u < 8; ++u)  // elements of the lanes past a head of 64 meet keys of zero
        raw[k][u] = *reinterpret_cast<const f32x4*>(x + k * 128 + (S::D < 128 ? quarter & 1 : quarter) * 32 + u * 4);
  }

  __device__ __forceinline__ void convert(float sign) {
#pragma unroll
    for (int k = 0; k < S::kKSteps; ++k)
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const float y = raw[k][j / 4][j % 4];
        float left = sign * y;
#pragma unroll
        for (int piece = 0; piece < 3; ++piece) {
          // bf16's largest number, where rounding would pass it; an infinity still leaves one
          w[k][j / 8][piece][j % 8] = (__bf16)(piece ? left : fminf(fmaxf(left, -kBf16Max), kBf16Max));
          left -= (float)w[k][j / 8][piece][j % 8];
        }
      }
  }

  static constexpr int kProducts = 12;
  __device__ __forceinline__ f32x4 product(int i, i32x4 codes, int scale, int k, f32x4 acc) const {
    const int piece = 2 - i / 4, u = i % 4;
    bf16x2 y[4];
    fp4_to_bf16x8((uint32_t)codes[u], (uint32_t)scale, y);
    u32x4 a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = scale == 255 ? 0x7FC07FC0u : __builtin_bit_cast(uint32_t, y[j]);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), w[k][u][piece], acc, 0, 0, 0);
  }
};

template <int N>
struct Blocks {
  static constexpr int value = N;
};

// One request's part in the line.  A row tile's length in it is the number of
// (token, query head of the group) pairs that its last row may see, and as much
// again as its beginning and end cost: with a mask the same for all tiles; a
// chain's tiles grow by kRows each.
template <typename S>
struct AttnReq {
  int len, rows, tiles;      // context, new rows, row tiles per kv head
  int64_t first, more, all;  // length of tile 0, growth, sum over the tiles

  __device__ __forceinline__ AttnReq(const KvAttnParams& p, int q) {
    const KvRows x = kv_rows(p.len, p.n, q, p.cap, p.max_blocks << p.c.page_shift);
    len = x.len, rows = x.rows;
    tiles = (rows * p.group + S::kRows - 1) / S::kRows;
    more = p.mask ? 0 : S::kRows;
    first = (int64_t)(len + S::kFixed) * p.group + (p.mask ? rows * p.group : S::kRows);
    all = before(tiles);
  }
  // All tiles as long as the longest.
  __device__ __forceinline__ void level() {
    first += more * (tiles - 1);
    more = 0;
    all = tiles * first;
  }
  // All tiles as long as the longest, up to whole pieces of `per`.
  __device__ __forceinline__ void pad(int64_t per) {
    level();
    first = (first + per - 1) / per * per;
    all = tiles * first;
  }
  // sum over the tiles before tile t
  __device__ __forceinline__ int64_t before(int t) const { return t * first + more * ((int64_t)t * (t - 1) / 2); }
  // the tile that holds place x < all
  __device__ __forceinline__ int tile_at(int64_t x) const {
    if (more == 0) return (int)(x / first);
    int lo = 0, hi = tiles - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before(mid) <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
  }
};

__device__ __forceinline__ void store4(float* out, f32x4 v) { *reinterpret_cast<f32x4*>(out) = v; }
__device__ __forceinline__ void store4(__bf16* out, f32x4 v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf16x4*>(out) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}

// Asks the scheduler for `products` matrix instructions with `others` vector
// instructions after each, in the straight piece of code that it stands in.
template <int PRODUCTS, int OTHERS>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < PRODUCTS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x2, OTHERS, 0);
  }
}

// Eight elements of a finished row m of (request, kv head), and its log-sum-exp.
template <typename TE, int D>
__device__ __forceinline__ void attn_out(const KvAttnParams& p, int q, int head, int m, int d, float top, float l,
                                         float r, const float (&y)[8]) {
  const int i = m / p.group, a = head * p.group + (m - i * p.group);
  const int64_t row = ((int64_t)q * p.cap + i) * p.q_heads + a;
  TE* out = static_cast<TE*>(p.out) + row * D + d;
  const float inv = r == 0.f ? 0.f : 1.f / r;
  if constexpr (sizeof(TE) == 2) {
    bf16x8 z;
#pragma unroll
    for (int k = 0; k < 8; ++k) z[k] = (__bf16)(y[k] * inv);
    *reinterpret_cast<bf16x8*>(out) = z;
  } else {
    f32x4 z0, z1;
#pragma unroll
    for (int k = 0; k < 4; ++k) z0[k] = y[k] * inv, z1[k] = y[k + 4] * inv;
    *reinterpret_cast<f32x4*>(out) = z0;
    *reinterpret_cast<f32x4*>(out + 4) = z1;
  }
  if (p.lse && d == 0) p.lse[row] = l == 0.f ? kNegInf : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

template <typename S>
__global__ __launch_bounds__(S::kThreads, S::kResident) __attribute__((amdgpu_waves_per_eu(S::kResident, S::kResident)))
void kv_attention_kernel(KvAttnParams p) {
  constexpr int D = S::D, MB = S::MB, WM = S::WM, WT = S::WT;
  using TE = typename S::TE;
  __shared__ __align__(16) char lds[S::kLds];
  __shared__ float m_lds[WT][S::kRows], l_lds[WT][S::kRows], r_lds[WT][S::kRows];
  __shared__ int64_t sum_lds[S::kThreads / 64];
  __shared__ int found;
  __shared__ int64_t found_at;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wt = wave / WM;
  const int col = lane & 15, quarter = lane >> 4;
  const int shift = p.c.page_shift, in_page = (1 << shift) - 1;

  // Of `pieces` of the line, the workgroup's: workgroups of one XCD (every eighth)
  // take neighbouring ones, so that row tiles of one request share its L2.
  const int groups = gridDim.x;
  auto own = [&](int pieces) {
    const int b = blockIdx.x, per_xcd = pieces / 8;
    return b < per_xcd * 8 ? (b % 8) * per_xcd + b / 8 : b;
  };
  int w;
  // Inclusive sum over a thread's request and those before it from q0 on.
  int64_t per = 0;  // length of a piece
  auto scan = [&](int q0, int64_t& v, int64_t& all) {
    v = 0;
    if (q0 + tid < p.R) {
      AttnReq<S> r(p, q0 + tid);
      if (p.spare) per ? r.pad(per) : r.level();
      v = r.all * p.c.heads;
    }
    int64_t incl = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t x = __shfl_up(incl, d);
      if (lane >= d) incl += x;
    }
    __syncthreads();
    if (lane == 63) sum_lds[wave] = incl;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int u = 0; u < S::kThreads / 64; ++u) {
      if (u < wave) incl += sum_lds[u];
      all += sum_lds[u];
    }
    return incl;
  };
  int q;
  int64_t at, begin, end;  // of request q's first step; the piece
  if (p.whole_tiles) {
    // short contexts: a tile a workgroup (of whole_tiles for each request and kv head)
    w = own(groups);
    q = w / (p.c.heads * p.whole_tiles);
    const int head = w / p.whole_tiles % p.c.heads, rt = w % p.whole_tiles;
    const AttnReq<S> r(p, q);
    if (rt >= r.tiles) return;
    at = -(head * r.all + r.before(rt));
    begin = 0, end = per = r.first + r.more * rt;
  } else {
    int64_t v, all, incl = scan(0, v, all), total = all;
    for (int q0 = S::kThreads; q0 < p.R; q0 += S::kThreads) {
      scan(q0, v, all);
      total += all;
    }
    const int64_t least = (int64_t)p.min_tokens * p.group;
    auto piece = [&](int n) { return (total + n - 1) / n; };  // of n
    per = piece(groups - p.spare);
    // few tiles of few steps: one workgroup a compute unit (fp32, 20000 tokens of one
    // row: 24.5 us with two, 21.2 with one; at eight steps a piece 38 and 42)
    if (S::kResident > 1 && p.spare && 2 * per < 5 * least) per = piece(groups / 2 - p.spare);
    per = max(per, least);
    if (p.spare) {
      // few tiles: each is padded to whole pieces, so that a workgroup has part of one
      total = 0;
      for (int q0 = 0; q0 < p.R; q0 += S::kThreads) {
        incl = scan(q0, v, all);
        total += all;
      }
    }
    w = own((int)((total + per - 1) / per));
    begin = per * w, end = min(begin + per, total);
    if (tid == 0) p.joins[w].q = -1;
    if (begin >= end) return;
    int64_t before = 0;
    for (int q0 = 0; q0 < p.R; q0 += S::kThreads) {
      if (p.R > S::kThreads) incl = scan(q0, v, all);
      if (before + incl - v <= begin && begin < before + incl) {
        found = q0 + tid;
        found_at = before + incl - v;
      }
      before += all;
    }
    __syncthreads();
    q = __builtin_amdgcn_readfirstlane(found);
    at = found_at;
  }

  const int g_rows = p.group;
  for (int64_t pos = begin; pos < end && q < p.R;) {
    AttnReq<S> r(p, q);
    if (p.spare) r.pad(per);
    if (pos >= at + r.all * p.c.heads) {
      at += r.all * p.c.heads;
      ++q;
      continue;
    }
    const int head = (int)((pos - at) / r.all);
    const int rt = r.tile_at(pos - at - head * r.all);
    const int64_t tile_at = at + head * r.all + r.before(rt), tile_len = r.first + r.more * rt, tile_end = tile_at + tile_len;
    const int rows_m = r.rows * g_rows, m0 = rt * S::kRows;
    const int context = r.len, all_tokens = r.len + r.rows;
    const int32_t* table = p.table + (size_t)q * p.max_blocks;

    // ---- tokens
    // Where waves share values, weights are taken with one rounding against maxima up
    // to kFused; a row that has seen no score above -inf yet counts as past that, so
    // that it looks for one in every half tile.
    constexpr float kFused = 4194304.f, kNone = WM > 1 ? 2.f * kFused : 0.f;  // 2^22
    float m_run[MB], m_neg[MB], l_run[MB], r_run[MB];  // the maximum, its negative (kNone for none), the sums of weights
    f32x4 o[MB][D / 16];
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      m_run[b] = kNegInf, m_neg[b] = kNone, l_run[b] = 0.f, r_run[b] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[b][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // last position that a row of the tile sees, and so the last step
    const int i_last = min((m0 + S::kRows - 1) / g_rows, r.rows - 1);
    const int need = p.mask ? all_tokens : context + i_last + 1;
    const int all_seen = p.mask ? context : context + m0 / g_rows + 1;  // what every row sees
    // the workgroup's steps: both sides of a cut round its place up alike
    const int64_t steps = (need + S::kTile * WT - 1) / (S::kTile * WT);
    const int64_t stop = min(end, tile_end);
    const int s0 = (int)(((pos - tile_at) * steps + tile_len - 1) / tile_len);
    const int s1 = (int)(((stop - tile_at) * steps + tile_len - 1) / tile_len);

    constexpr int kVLoads = D / 32;  // of a token tile, 16 bytes a lane
    constexpr int kVMine = (kVLoads + WM - 1) / WM;
    i32x4 kc[4][S::kKSteps];  // keys: codes and scales of the lane's token in each run of 16
    int ks[4][S::kKSteps];
    u32x4 vc[kVMine];         // values
    uint32_t vs[kVMine];
    // The table's entries of a tile's runs of tokens, looked at a step before
    // they are used (a check next to the load would wait for it), and the pages
    // they name, -1 where there is none.
    constexpr int kRuns = S::kRuns;
    auto look_up = [&](int step, int (&entry)[kRuns]) {
      const int b0 = ((step * WT + wt) * S::kTile) >> shift;
#pragma unroll
      for (int u = 0; u < kRuns; ++u) entry[u] = table[min(b0 + (16 * u >> shift), p.max_blocks - 1)];
    };
    auto pages_of = [&](int step, const int (&entry)[kRuns], int (&pg)[kRuns]) {
      const int b0 = ((step * WT + wt) * S::kTile) >> shift;
#pragma unroll
      for (int u = 0; u < kRuns; ++u) {
        const int page = __builtin_amdgcn_readfirstlane(entry[u]);
        pg[u] = b0 + (16 * u >> shift) < p.max_blocks && (uint32_t)page < (uint32_t)p.c.num_pages ? page : -1;
      }
    };
    // Loads of runs without a page go to page 0 and are set aside: keys get
    // scale 255, so that their scores are not-a-number, values read as zero.
    auto load_keys = [&](int step, const int (&pg)[kRuns], int half = -1) {  // 0, 2: of runs 0, 1 or 2, 3 alone
      const int t0 = (step * WT + wt) * S::kTile;
      const int part = D >= 128 ? quarter : quarter & 1;
      const int lane_code = col * (D / 2) + part * 16, lane_scale = col * (D / 32) + part;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (half >= 0 && (u & 2) != half) continue;
        const int run = kRuns == 1 ? 0 : u, off = (t0 + 16 * run) & in_page, more_off = kRuns == 1 ? 16 * u : 0;
        const char* blk = kv_block<D>(p.c, max(pg[run], 0), head);
        const char* codes = blk + KvBlock<D>::key_codes(off);
        const char* scales = blk + KvBlock<D>::key_scales(off, shift);
#pragma unroll
        for (int k = 0; k < S::kKSteps; ++k) {
          kc[u][k] = *reinterpret_cast<const i32x4*>(codes + (uint32_t)lane_code + (more_off * (D / 2) + k * 64));
          ks[u][k] = *reinterpret_cast<const uint8_t*>(scales + (uint32_t)lane_scale + (more_off * (D / 32) + k * 4));
        }
      }
    };
    // the page of the lane's part of load j: a load covers 2048 / D tokens, half of
    // a run of 16, one or two
    auto value_page = [&](int j, const int (&pg)[kRuns]) {
      if constexpr (kRuns == 1) {
        return pg[0];
      } else if constexpr (D == 64) {
        const int page = lane < 32 ? pg[0] : pg[1];
        return j * WM + wm ? (lane < 32 ? pg[2] : pg[3]) : page;
      } else {
        const int run = min((j * WM + wm) * 128 / D, 3);
        return run == 0 ? pg[0] : run == 1 ? pg[1] : run == 2 ? pg[2] : pg[3];
      }
    };
    auto load_values = [&](int step, const int (&pg)[kRuns]) {
      const int t0 = (step * WT + wt) * S::kTile;
#pragma unroll
      for (int j = 0; j < kVMine; ++j) {
        if (j * WM + wm < kVLoads) {
          const int piece = (j * WM + wm) * 64 + lane;  // in the tile's 2 D pieces of 32 elements
          const int tok = piece / (D / 32), part = piece % (D / 32);
          if constexpr (kRuns == 1) {
            const int off = t0 & in_page;
            const char* blk = kv_block<D>(p.c, max(pg[0], 0), head);
            vc[j] = *reinterpret_cast<const u32x4*>(blk + KvBlock<D>::value_codes(off, shift) + (uint32_t)(piece * 16));
            vs[j] = *reinterpret_cast<const uint8_t*>(blk + KvBlock<D>::value_scales(off, shift) + (uint32_t)piece);
          } else {
            const int page = value_page(j, pg);
            const int off = (t0 + tok) & in_page;
            const char* blk = kv_block<D>(p.c, max(page, 0), head);
            vc[j] = *reinterpret_cast<const u32x4*>(blk + (uint32_t)(KvBlock<D>::value_codes(off, shift) + part * 16));
            vs[j] = *reinterpret_cast<const uint8_t*>(blk + (uint32_t)(KvBlock<D>::value_scales(off, shift) + part));
          }
        }
      }
    };
    // unpack a load's values into LDS, at the tile's token `tok - first`
    auto unpack = [&](int j, const int (&pg)[kRuns], char* to, int first) {
      const int piece = (j * WM + wm) * 64 + lane;
      const int tok = piece / (D / 32) - first, part = piece % (D / 32);
      if (j * WM + wm >= kVLoads) return;
      const uint32_t sc = value_scale(vs[j]);
      const bool none = vs[j] == 255 || value_page(j, pg) < 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        bf16x2 y[4];
        fp4_to_bf16x8(none ? 0u : vc[j][u], sc, y);
        u32x4 z;
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] = __builtin_bit_cast(uint32_t, y[k]);
        *reinterpret_cast<u32x4*>(to + tok * S::kVRow + part * 64 + u * 16) = z;
      }
    };

    // Each register is loaded again for the next step as soon as this one is
    // done with it; pages are looked up a step earlier.
    // Where waves share the values, they are unpacked a step before they are
    // used: their loads run a step ahead of the keys'.
    constexpr int kAhead = WM > 1 ? 1 : 0;
    int pg[2 + kAhead][kRuns], entry[kRuns];  // pages of step s (while s + 1 is loaded), s + 1, s + 2
    look_up(s0, entry);
    // queries: those of rows past the last read row 0 and are of no use
    AttnQuery<S> qp[MB];
    // what <Q, K> is multiplied by to give base-2 units, queries with the scale's sign; a scale of
    // 0 is one of 1 on queries of 0, so that a hidden score's -inf stays one
    const float sign = p.scale_log2 == 0.f ? 0.f : p.scale_log2 < 0.f ? -1.f : 1.f;
    const float unit = p.scale_log2 == 0.f ? 1.f : __builtin_fabsf(p.scale_log2);
    int row_i[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      const int m = m0 + (b * WM + wm) * 16 + col;
      const bool there = m < rows_m;
      const int i = there ? m / g_rows : 0, g = there ? m - i * g_rows : 0;
      row_i[b] = there ? i : -1;
      if (WM > 1 && !there) m_run[b] = 0.f, m_neg[b] = 0.f;
      qp[b].fetch(static_cast<const TE*>(p.q) + ((int64_t)q * p.cap + i) * p.q_stride + (int64_t)(head * g_rows + g) * D, quarter);
    }
    pages_of(s0, entry, pg[0]);
    load_keys(s0, pg[0]);
    load_values(s0, pg[0]);
    if constexpr (kAhead) {
      look_up(s0 + 1, entry);
      pages_of(s0 + 1, entry, pg[1]);
    }
    look_up(s0 + 1 + kAhead, entry);

#pragma unroll
    for (int b = 0; b < MB; ++b) qp[b].convert(sign);

    char* v_lds = lds + wt * (S::kVTokens * S::kVRow);
    constexpr int kGroups = D / 64;  // of four blocks of 16 elements
    // Scores of runs u0... of the keys in registers, on the pages `pg`.
    auto score = [&](auto& x, int u0, const int (&pg_)[kRuns]) {
      constexpr int NB = sizeof(x) / sizeof(x[0]), N = sizeof(x[0]) / sizeof(x[0][0]);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int u = 0; u < N; ++u) x[b][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < S::kKSteps; ++k)
#pragma unroll
        for (int i = 0; i < AttnQuery<S>::kProducts; ++i)
#pragma unroll
          for (int u = 0; u < N; ++u) {
            i32x4 codes = kc[u0 + u][k];
            if (D < 128 && quarter >= 2) codes = i32x4{0, 0, 0, 0};
            const int scale = pg_[kRuns == 1 ? 0 : u0 + u] < 0 ? 255 : ks[u0 + u][k];
#pragma unroll
            for (int b = 0; b < NB; ++b) x[b][u] = qp[b].product(i, codes, scale, k, x[b][u]);
          }
    };
    // -inf for what a row does not see, of runs u0... of the tile at t0.
    auto hide = [&](auto& x, int u0, int t0) {
      constexpr int NB = sizeof(x) / sizeof(x[0]), N = sizeof(x[0]) / sizeof(x[0][0]);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        uint64_t sees = 0;
        const int i = row_i[b], j0 = t0 - context;
        if (i >= 0) {
          if (!p.mask) {
            const int cnt = min(max(i + 1 - j0, 0), 64);
            sees = cnt == 64 ? ~0ull : (1ull << cnt) - 1;
          } else if (t0 < all_tokens) {
            const uint32_t* bits = p.mask + ((size_t)q * p.cap + i) * p.mask_words;
            const int first = max(j0, 0), w0 = first >> 5, sh = first & 31;
            uint32_t word[3];
#pragma unroll
            for (int u = 0; u < 3; ++u) word[u] = bits[min(w0 + u, p.mask_words - 1)];  // what repeats lies past all rows
            uint64_t win = (((uint64_t)word[1] << 32) | word[0]) >> sh;
            if (sh) win |= (uint64_t)word[2] << (64 - sh);
            if (j0 < 0) win = j0 > -64 ? (win << -j0) | ((1ull << -j0) - 1) : ~0ull;
            const int cnt = min(all_tokens - t0, 64);
            sees = cnt >= 64 ? win : win & ((1ull << cnt) - 1);
          }
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
          const uint32_t four = (uint32_t)(sees >> (16 * (u0 + u) + 4 * quarter)) & 15u;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[b][u][e] = four >> e & 1 ? x[b][u][e] : kNegInf;
        }
      }
    };
    auto highest = [&](const auto& x, auto& top) {
      constexpr int NB = sizeof(x) / sizeof(x[0]), N = sizeof(x[0]) / sizeof(x[0][0]);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        top[b] = kNegInf;
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) top[b] = fmaxf(top[b], x[b][u][e]);
        top[b] = fmaxf(top[b], xor16_f32(top[b]));
        top[b] = fmaxf(top[b], xor32_f32(top[b])) * unit;
      }
    };
    // Raises what weights are taken against to the maximum `top`, which it may lag
    // behind by 2^8, so that most tiles rescale nothing.
    auto rescale = [&](const auto& top) {
      constexpr int NB = sizeof(top) / sizeof(top[0]);
      bool rises = false;
#pragma unroll
      for (int b = 0; b < NB; ++b) rises |= top[b] > m_run[b] + 8.f;
      if (__any(rises))
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const float m_new = fmaxf(m_run[b], top[b]);
          const float keep = m_new == kNegInf ? 1.f : exp2_fast(m_run[b] - m_new);
          m_run[b] = m_new;
          m_neg[b] = m_new == kNegInf ? kNone : -m_new;
          l_run[b] *= keep;
          r_run[b] *= keep;
#pragma unroll
          for (int d = 0; d < D / 16; ++d) o[b][d] *= keep;
        }
    };
    // Weights of two runs as the products' B operand, and their sums: as they are
    // for the log-sum-exp, and as the products take them, which is what outputs are
    // divided by, so that the rounding of a row's large weights cancels.
    // `fused`: with one rounding instead of two.  The maximum was rounded when it was
    // taken times `unit`: a weight against it is then off by a factor of up to
    // 2^(|m| 2^-24), the same for all of a row, which must not be large.
    auto weigh = [&](const auto& x, int u0, auto& w8, auto& sum, auto& rsum, bool fused) {
      constexpr int NB = sizeof(x) / sizeof(x[0]);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        sum[b] = 0.f;
        rsum[b] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float left = exp2_fast(fused ? __builtin_fmaf(x[b][u0 + e / 4][e % 4], unit, m_neg[b])
                                       : x[b][u0 + e / 4][e % 4] * unit + m_neg[b]);
          sum[b] += left;
#pragma unroll
          for (int piece = 0; piece < S::kP; ++piece) {
            w8[b][piece][e] = (__bf16)left;
            left -= (float)w8[b][piece][e];
          }
        }
        // computed here, beside the products, and not where they are used
#pragma unroll
        for (int piece = 0; piece < S::kP; ++piece) {
          u32x4 bits = __builtin_bit_cast(u32x4, w8[b][piece]);
          asm volatile("" : "+v"(bits));
          w8[b][piece] = __builtin_bit_cast(bf16x8, bits);
        }
        if constexpr (S::kP == 1) {
          const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
          for (int e = 0; e < 8; e += 2)
            rsum[b] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w8[b][0][e], w8[b][0][e + 1]}, ones, rsum[b], false);
        }
      }
    };
    // Values of a half tile at `from` as the products' A operand, and the products.
    s16x8 va[2][4];
    auto read_group = [&](const char* from, int g) {
      typedef __attribute__((address_space(3))) s16x4* lds_ptr;
      const char* at = from + (4 * quarter + col / 4) * S::kVRow + (col % 4) * 8 + g * 128;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + x * 32));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + x * 32 + 16 * S::kVRow));
        va[g & 1][x] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    };
    auto add_group = [&](int g, const auto& w8) {
      constexpr int NB = sizeof(w8) / sizeof(w8[0]);
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int piece = S::kP - 1; piece >= 0; --piece)
            o[b][4 * g + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va[g & 1][x]), w8[b][piece],
                                                                      o[b][4 * g + x], 0, 0, 0);
    };

    if constexpr (WM == 1) {
      // each wave on its own: bound by the bytes that are on their way
      for (int s = s0; s < s1; ++s) {
        const int t0 = (s * WT + wt) * S::kTile;
        const bool more = s + 1 < s1;
        pages_of(s + 1, entry, pg[1]);
        look_up(s + 2, entry);
        if (t0 < need) {
          f32x4 sc[MB][4];
          score(sc, 0, pg[0]);
          if (more) load_keys(s + 1, pg[1]);
          if (t0 + S::kTile > all_seen) hide(sc, 0, t0);
          float top[MB];
          highest(sc, top);
          rescale(top);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int j = 0; j < kVMine / 2; ++j) unpack(half * (kVMine / 2) + j, pg[0], v_lds, half * 32);
            if (half == 1 && more) load_values(s + 1, pg[1]);
            bf16x8 w8[MB][S::kP];
            float sum[MB], rsum[MB];
            weigh(sc, 2 * half, w8, sum, rsum, false);
#pragma unroll
            for (int b = 0; b < MB; ++b) l_run[b] += sum[b], r_run[b] += rsum[b];
            wave_lds_sync();
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
              read_group(v_lds, g);
              add_group(g, w8);
            }
            wave_lds_sync();
          }
        }
#pragma unroll
        for (int u = 0; u < kRuns; ++u) pg[0][u] = pg[1][u];
      }
    } else {
      // Bound by instructions: a wave's products and its softmax alternate by half
      // tiles so that one runs under the other: while a half is scored, the half
      // before it becomes weights, whose products run beside the loads' work.
      // The maximum is found for the first half and where rows differ in what they
      // see; elsewhere weights are taken against what there is, and only where a sum
      // of them passes kMost is the maximum found and the half weighed again.  (Any
      // reference serves as long as nothing overflows: fp32 sums and bf16 weights
      // are as exact at 2^12 as at 1.)  Weights are taken with one fused operation (two:
      // prompts of 8000 rows 695 us, this 650), but beyond scores of 2^22 with two.  Values lie in a ring of three tiles: the one that
      // is unpacked, the one at hand and the one whose second half is still due.
      constexpr int kSlot = 64 * S::kVRow;
      int cur = 0, before = 0;
#pragma unroll
      for (int j = 0; j < kVMine; ++j) unpack(j, pg[0], v_lds, 0);
      load_values(s0 + 1, pg[1]);
      if (m0 + wm * 16 >= rows_m) {
        // no rows for this wave: it unpacks its share of the values
        __syncthreads();
        for (int s = s0; s < s1; ++s) {
          const int next = cur == 2 * kSlot ? 0 : cur + kSlot;
          pages_of(s + 2, entry, pg[2]);
          look_up(s + 3, entry);
#pragma unroll
          for (int j = 0; j < kVMine; ++j) unpack(j, pg[1], v_lds + next, 0);
          load_values(s + 2, pg[2]);
          __syncthreads();
          cur = next;
#pragma unroll
          for (int u = 0; u < kRuns; ++u) pg[1][u] = pg[2][u];
        }
      } else {
        // with the blocks of 16 rows that the wave has
        auto run = [&](auto blocks) {
          constexpr int NB = decltype(blocks)::value;
          f32x4 sc[2][NB][2];
          bf16x8 w8[2][NB][S::kP];
  #pragma unroll
          for (int b = 0; b < NB; ++b)
  #pragma unroll
            for (int piece = 0; piece < S::kP; ++piece)
  #pragma unroll
              for (int e = 0; e < 8; ++e) w8[1][b][piece][e] = (__bf16)0.f;
          float sum[NB], rsum[NB];
          constexpr float kMost = 4096.f;
          auto raise = [&](auto& x, int u0, int t0, bool part) {
            if (part) hide(x, u0, t0);
            float top[NB];
            highest(x, top);
            rescale(top);
          };
          // The products are issued before this point, not behind the branch that follows
          // (no instruction: nothing waits for their results).
          auto stay = [&](f32x4 (&x)[NB][2]) {
  #pragma unroll
            for (int b = 0; b < NB; ++b) asm volatile("" : "+v"(x[b][0]), "+v"(x[b][1]));
          };
          auto settle = [&](auto& x, int u0, int t0, bf16x8 (&w)[NB][S::kP]) {
            bool over = false;
  #pragma unroll
            for (int b = 0; b < NB; ++b) over |= sum[b] > kMost || __builtin_fabsf(m_neg[b]) > kFused;
            if (__any(over)) {
              raise(x, u0, t0, false);  // hidden already
              weigh(x, 0, w, sum, rsum, false);
            }
  #pragma unroll
            for (int b = 0; b < NB; ++b) l_run[b] += sum[b], r_run[b] += rsum[b];
          };
          score(sc[0], 0, pg[0]);
          __syncthreads();
          read_group(v_lds + 32 * S::kVRow, 0);  // multiplied with weights of zero
          for (int s = s0; s < s1; ++s) {
            const int t0 = (s * WT + wt) * S::kTile;
            const bool part = t0 + S::kTile > all_seen;
            const int next = cur == 2 * kSlot ? 0 : cur + kSlot;
            pages_of(s + 2, entry, pg[2]);
            look_up(s + 3, entry);
            const bool first = part || s == s0;
            // Two workgroups share a compute unit, and the older one's waves always go
            // first: it ended at 580 us where the other needed 740.  They take turns at a
            // higher priority instead, 41 us each by the device's clock (prompts of 8000 rows: 690 us, in turn 650).
            if ((uint32_t)__builtin_readsteadycounter() >> 12 & 1 ^ (blockIdx.x >= gridDim.x / 2)) __builtin_amdgcn_s_setprio(1);
            else __builtin_amdgcn_s_setprio(0);
            // What is loaded past the last tile lies in some page and is of no use; a
            // branch around it would keep the products from running beside the rest.
            // second half of the tile before, first half's weights, second half's scores
            load_keys(s + 1, pg[1], 0);
  #pragma unroll
            for (int g = 0; g < kGroups; ++g) {
              if (g + 1 < kGroups) read_group(v_lds + before + 32 * S::kVRow, g + 1);
              add_group(g, w8[1]);
            }
            interleave<NB * S::kP * D / 16, 2>();
            if (first) raise(sc[0], 0, t0, part);
            read_group(v_lds + cur, 0);
            score(sc[1], 2, pg[0]);
            weigh(sc[0], 0, w8[0], sum, rsum, true);
            stay(sc[1]);
            interleave<NB * 2 * AttnQuery<S>::kProducts * S::kKSteps, 8>();
            settle(sc[0], 0, t0, w8[0]);
            // first half of this tile, second half's weights, the next tile's scores
            load_keys(s + 1, pg[1], 2);
  #pragma unroll
            for (int g = 0; g < kGroups; ++g) {
              if (g + 1 < kGroups) read_group(v_lds + cur, g + 1);
              add_group(g, w8[0]);
            }
  #pragma unroll
            for (int j = 0; j < kVMine; ++j) unpack(j, pg[1], v_lds + next, 0);
            load_values(s + 2, pg[2]);
            interleave<NB * S::kP * D / 16, 4>();
            if (first) raise(sc[1], 2, t0, part);
            read_group(v_lds + cur + 32 * S::kVRow, 0);
            score(sc[0], 0, pg[1]);
            weigh(sc[1], 0, w8[1], sum, rsum, true);
            stay(sc[0]);
            interleave<NB * 2 * AttnQuery<S>::kProducts * S::kKSteps, 8>();
            settle(sc[1], 2, t0, w8[1]);
            __syncthreads();  // the next tile's values are there, those before this one's are done with
            before = cur;
            cur = next;
  #pragma unroll
            for (int u = 0; u < kRuns; ++u) pg[0][u] = pg[1][u], pg[1][u] = pg[2][u];
          }
  #pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            if (g + 1 < kGroups) read_group(v_lds + before + 32 * S::kVRow, g + 1);
            add_group(g, w8[1]);
          }
        };
        if (MB > 1 && m0 + (WM + wm) * 16 >= rows_m) run(Blocks<1>{});
        else run(Blocks<MB>{});
      }
    }

    // ---- join the waves, and out
    const bool whole = pos == tile_at && stop == tile_end;
    const int slot = 2 * w + (pos == begin ? 0 : 1);
    if constexpr (WT == 1) {
      // a wave has all of its rows: four elements a lane
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        const float l = cross_row_sum(l_run[b]), r = S::kP == 1 ? cross_row_sum(r_run[b]) : l;
        const int m_in = (b * WM + wm) * 16 + col;
        if (row_i[b] < 0) continue;
        if (whole) {
          const int64_t row = ((int64_t)q * p.cap + row_i[b]) * p.q_heads + head * g_rows + (m0 + m_in - row_i[b] * g_rows);
          const float inv = r == 0.f ? 0.f : 1.f / r;
#pragma unroll
          for (int d = 0; d < D / 16; ++d) store4(static_cast<TE*>(p.out) + row * D + d * 16 + quarter * 4, o[b][d] * inv);
          if (p.lse && quarter == 0) p.lse[row] = l == 0.f ? kNegInf : (m_run[b] + __builtin_amdgcn_logf(l)) * kLn2;
        } else {
          float* part = p.parts + ((size_t)slot * S::kRows + m_in) * D + quarter * 4;
#pragma unroll
          for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4*>(part + d * 16) = o[b][d];
          if (quarter == 0) p.stats[(size_t)slot * S::kRows + m_in] = AttnStat{m_run[b], l, r, 0.f};
        }
      }
      __syncthreads();  // values in LDS have been read
    } else {
      __syncthreads();  // values in LDS have been read
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        l_run[b] = cross_row_sum(l_run[b]);
        r_run[b] = S::kP == 1 ? cross_row_sum(r_run[b]) : l_run[b];
        if (quarter == 0) {
          m_lds[wt][(b * WM + wm) * 16 + col] = m_run[b];
          l_lds[wt][(b * WM + wm) * 16 + col] = l_run[b];
          r_lds[wt][(b * WM + wm) * 16 + col] = r_run[b];
        }
      }
      __syncthreads();
      float* o_lds = reinterpret_cast<float*>(lds);
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        const int mine_row = (b * WM + wm) * 16 + col;
        float top = kNegInf;
#pragma unroll
        for (int u = 0; u < WT; ++u) top = fmaxf(top, m_lds[u][mine_row]);
        const float keep = top == kNegInf ? 1.f : exp2_fast(m_run[b] - top);
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
          *reinterpret_cast<f32x4*>(o_lds + ((wt * WM + wm) * 16 + col) * S::kORow + d * 16 + quarter * 4) = o[b][d] * keep;
        __syncthreads();
        for (int x = tid; x < WM * 16 * (D / 8); x += S::kThreads) {
          const int row = x / (D / 8), d = x % (D / 8) * 8;  // row: of the waves' blocks b
          const int m_in = (b * WM + row / 16) * 16 + row % 16, m = m0 + m_in;
          if (m >= rows_m) continue;
          float top2 = kNegInf;
#pragma unroll
          for (int u = 0; u < WT; ++u) top2 = fmaxf(top2, m_lds[u][m_in]);
          float l = 0.f, r = 0.f, y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int u = 0; u < WT; ++u) {
            const float keep_u = top2 == kNegInf ? 1.f : exp2_fast(m_lds[u][m_in] - top2);
            l += l_lds[u][m_in] * keep_u;
            r += r_lds[u][m_in] * keep_u;
            const float* z = o_lds + (u * WM * 16 + row) * S::kORow + d;
            const f32x4 z0 = *reinterpret_cast<const f32x4*>(z), z1 = *reinterpret_cast<const f32x4*>(z + 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] += z0[k], y[k + 4] += z1[k];
          }
          if (whole) {
            attn_out<TE, D>(p, q, head, m, d, top2, l, r, y);
          } else {
            float* part = p.parts + ((size_t)slot * S::kRows + m_in) * D + d;
            *reinterpret_cast<f32x4*>(part) = f32x4{y[0], y[1], y[2], y[3]};
            *reinterpret_cast<f32x4*>(part + 4) = f32x4{y[4], y[5], y[6], y[7]};
            if (d == 0) p.stats[(size_t)slot * S::kRows + m_in] = AttnStat{top2, l, r, 0.f};
          }
        }
        __syncthreads();
      }
    }
    // the first workgroup whose piece begins inside the tile says where its parts are
    if (tid == 0 && pos == begin && begin > tile_at && begin - per <= tile_at)
      p.joins[w] = AttnJoin{q, head, m0, min(S::kRows, rows_m - m0), 2 * (w - 1) + (begin - per == tile_at ? 0 : 1),
                            (int)((tile_end - 1) / per)};
    pos = stop;
  }
}

// Joins the parts of the tiles that more than one workgroup worked on.  A unit
// is ROWS rows of the tile that joins[w] names (most name none): a block looks at
// 64 units at once and takes those it finds one by one.  D / 4 lanes hold a row
// and go through its parts with a running maximum; where a block has more
// threads than that, groups of them take parts in turn (small tiles are cut into
// many) and are joined in LDS.
template <typename TE, int D, int THREADS, int ROWS>
__global__ __launch_bounds__(THREADS) void kv_join_kernel(KvAttnParams p, int rows_shift, int pieces) {
  constexpr int kLanes = D / 4, kGroups = THREADS / (ROWS * kLanes), kBatch = 8, kUnit = __builtin_ctz(ROWS);
  __shared__ __align__(16) f32x4 o_lds[kGroups > 1 ? kGroups : 1][ROWS][kLanes];
  __shared__ AttnStat s_lds[kGroups][ROWS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int row = tid / kLanes % ROWS, grp = tid / kLanes / ROWS, at = tid % kLanes;
  // the pieces' first rows, then their next ones, ..., each turned a little, so
  // that few tiles of many rows spread over the blocks
  const int units = pieces << (rows_shift - kUnit);
  auto piece_of = [&](int unit) { return (unit + unit / pieces * 61) % pieces; };
  for (int u0 = blockIdx.x; u0 < units; u0 += 64 * gridDim.x) {
    const int mine = u0 + lane * (int)gridDim.x;
    AttnJoin found = {-1, 0, 0, 0, 0, 0};
    if (mine < units) found = p.joins[piece_of(mine)];
    const bool on = found.q >= 0 && (mine / pieces << kUnit) < found.rows;
    for (uint64_t left = __ballot(on); left; left &= left - 1) {
      const int bit = __builtin_ctzll(left), unit = u0 + bit * (int)gridDim.x, w = piece_of(unit);
      const int first = lane_i32(found.first, bit), count = lane_i32(found.last, bit) - w + 2;
      const int row_in = (unit / pieces << kUnit) + row;
      // the row of part x: the first, then those of slots 2 w, 2 (w + 1), ...
      auto place = [&](int x) { return ((size_t)(x ? 2 * (w + x - 1) : first) << rows_shift) + row_in; };
      float top = kNegInf, l = 0.f, r = 0.f;
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
      for (int x0 = grp; x0 < count; x0 += kBatch * kGroups) {
        f32x4 part[kBatch];
        AttnStat st[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
          if (x0 + b * kGroups < count) {
            const size_t from = place(x0 + b * kGroups);
            part[b] = *reinterpret_cast<const f32x4*>(p.parts + from * D + at * 4);
            st[b] = p.stats[from];
          } else {
            part[b] = f32x4{0.f, 0.f, 0.f, 0.f};
            st[b] = AttnStat{kNegInf, 0.f, 0.f, 0.f};
          }
        float high = top;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) high = fmaxf(high, st[b].m);
        const float sub = high == kNegInf ? 0.f : high, old = exp2_fast(top - sub);
        l *= old;
        r *= old;
        y *= old;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const float keep = st[b].m == kNegInf ? 1.f : exp2_fast(st[b].m - sub);  // a row of not-a-numbers has no maximum
          l += st[b].l * keep;
          r += st[b].r * keep;
          y += part[b] * keep;
        }
        top = high;
      }
      if constexpr (kGroups > 1) {
        __syncthreads();  // the unit before has been read
        o_lds[grp][row][at] = y;
        if (at == 0) s_lds[grp][row] = AttnStat{top, l, r, 0.f};
        __syncthreads();
        if (grp == 0) {
          float high = kNegInf;
#pragma unroll
          for (int g = 0; g < kGroups; ++g) high = fmaxf(high, s_lds[g][row].m);
          l = 0.f, r = 0.f, y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            const AttnStat st = s_lds[g][row];
            const float keep = st.m == kNegInf ? 1.f : exp2_fast(st.m - high);
            l += st.l * keep;
            r += st.r * keep;
            y += o_lds[g][row][at] * keep;
          }
          top = high;
        }
      }
      if (grp == 0 && row_in < lane_i32(found.rows, bit)) {
        const int m = lane_i32(found.m0, bit) + row_in, i = m / p.group;
        const int64_t out_row = ((int64_t)lane_i32(found.q, bit) * p.cap + i) * p.q_heads + lane_i32(found.head, bit) * p.group + (m - i * p.group);
        store4(static_cast<TE*>(p.out) + out_row * D + at * 4, y * (r == 0.f ? 0.f : 1.f / r));
        if (p.lse && at == 0) p.lse[out_row] = l == 0.f ? kNegInf : (top + __builtin_amdgcn_logf(l)) * kLn2;
      }
    }
  }
}

}  // namespace ts
