// C ABI of the target's 4-bit key-value cache (treespark_kv.h): argument checks and launches.
#include <cmath>

#include "host_api.hpp"
#include "kv_launch.hpp"

namespace ts {
namespace {

constexpr int kMaxRequests = 65536;
constexpr int kMaxGroup = 256;  // (2^30 tokens of 256 heads) * 2^24 steps: places in the attention's line stay in 64 bits
constexpr int64_t kMaxElements = (int64_t)1 << 34;  // of rows in one call: 2^31 threads

bool page_size_ok(int32_t p) { return p == 16 || p == 32 || p == 64 || p == 128 || p == 256; }
bool head_dim_ok(int32_t d) { return d == 64 || d == 128 || d == 256; }
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int32_t check_cache(const ts_kv_cache* c) {
  if (!c) return fail(TS_EINVAL, "cache is NULL");
  if (!c->pages) return fail(TS_EINVAL, "cache pages pointer is NULL");
  if (c->layers < 1 || c->num_pages < 1 || c->heads < 1)
    return fail(TS_EINVAL, "cache sizes must be positive (layers=%d num_pages=%d heads=%d)", c->layers, c->num_pages, c->heads);
  if (!page_size_ok(c->page_size)) return fail(TS_EUNSUPPORTED, "page_size=%d is not 16, 32, 64, 128 or 256", c->page_size);
  if (!head_dim_ok(c->head_dim)) return fail(TS_EUNSUPPORTED, "head_dim=%d is not 64, 128 or 256", c->head_dim);
  if ((int64_t)c->num_pages * c->page_size >= (int64_t)1 << 31)
    return fail(TS_EUNSUPPORTED, "num_pages * page_size = %lld reaches 2^31", (long long)c->num_pages * c->page_size);
  if (c->layers > 65535 || c->heads > 65536) return fail(TS_EUNSUPPORTED, "layers=%d or heads=%d out of range", c->layers, c->heads);
  if (!aligned16(c->pages) || c->page_stride % 16 || c->layer_stride % 16)
    return fail(TS_EINVAL, "cache pages and strides must be multiples of 16 bytes");
  const int64_t block = (int64_t)c->heads * (int64_t)ts_kv_block_bytes(c->page_size, c->head_dim);
  if (c->page_stride < block) return fail(TS_EINVAL, "page_stride %lld < %lld bytes of a page", (long long)c->page_stride, (long long)block);
  if (c->layers > 1 && c->layer_stride < block)
    return fail(TS_EINVAL, "layer_stride %lld < %lld bytes of a page", (long long)c->layer_stride, (long long)block);
  return TS_OK;
}

int32_t check_layer(const ts_kv_cache* c, int32_t layer, int32_t layers) {
  if (layer < 0 || layers < 1 || layer > c->layers - layers)
    return fail(TS_EINVAL, "layers [%d, %lld) outside [0, %d)", layer, (long long)layer + layers, c->layers);
  return TS_OK;
}

int32_t check_dtype(int32_t dtype) {
  if (dtype != TS_F32 && dtype != TS_BF16) return fail(TS_EINVAL, "unknown dtype %d", dtype);
  return TS_OK;
}

int32_t check_requests(int32_t R, int32_t max_blocks, int32_t page_size) {
  if (R < 0) return fail(TS_EINVAL, "R=%d is negative", R);
  if (R > kMaxRequests) return fail(TS_EUNSUPPORTED, "R=%d exceeds %d", R, kMaxRequests);
  if (max_blocks < 1) return fail(TS_EINVAL, "max_blocks=%d", max_blocks);
  if ((int64_t)max_blocks * page_size > (int64_t)1 << 30)
    return fail(TS_EUNSUPPORTED, "max_blocks * page_size = %lld exceeds 2^30", (long long)max_blocks * page_size);
  if ((int64_t)R * max_blocks >= (int64_t)1 << 31)
    return fail(TS_EUNSUPPORTED, "R * max_blocks = %lld reaches 2^31", (long long)R * max_blocks);
  return TS_OK;
}

int log2i(int x) { return __builtin_ctz((unsigned)x); }

KvView view(const ts_kv_cache* c, int32_t layer) {
  return {static_cast<char*>(c->pages) + (int64_t)layer * c->layer_stride, c->layer_stride, c->page_stride,
          c->num_pages, log2i(c->page_size), c->heads};
}

// What a launch of the attention takes: the row tile, the workgroups, and where
// their partial results lie in the workspace.
struct AttnPlan {
  AttnTile tile;
  int rows, groups, min_tokens, spare, whole_tiles;
  size_t stats, joins, bytes;  // offsets after the parts, and all
};

// tokens: the most that a request's table can name (0: unknown, which takes the
// most workspace).
//
// The tile: the smallest that holds all rows of a request and kv head, so that its
// keys and values are read once, up to the largest, whose waves share them (64
// trees of up to 65 rows and 4 query heads a kv head over 500 to 8000 tokens: tiles
// of 128 rows 188 us, of 32 257, of 16 304; of 12 rows: 89 us, 119 in tiles of 32; of
// 7 rows: 80 either way, 90 in tiles of 16).  A few tiles cut into many pieces
// cost more in partial results than they gain, unless their context is long: one
// such tree over 5003 tokens took 40 us in tiles of 128 and 34 in tiles of 32,
// three of 33 rows in fp32 over 50 to 700 27 us in tiles of 64 and 21 in tiles of 16.
// Up to 64 rows that holds for long contexts too (one tree of 12 rows over 30000
// tokens: tiles of 32 29 us, of 128 36; four of 9 rows over 20000: 48 and 45).
//
// The workgroups: what a compute unit holds of them, so that none waits.  Tiles of
// 16 rows would allow three, which is better where a unit has a tile or more (1024
// tiles over 300 to 16000 tokens: 128 us with two, 124 with three; 256: 42.5 and 41.8;
// 128 over 16000: 67 and 72; 8 over 131001: 38 and 41).
AttnPlan attn_plan(const ts_kv_cache* c, int32_t R, int32_t cap, int32_t q_heads, int32_t dtype, int64_t tokens, int cus) {
  AttnPlan x;
  const int64_t rows = (int64_t)cap * (q_heads / c->heads), most = dtype == TS_F32 ? 64 : 128;
  const int64_t pairs = (int64_t)R * c->heads;  // of requests and kv heads
  const bool brief = tokens > 0 && tokens <= 16384 && pairs * ((rows + most - 1) / most) * 4 < cus;
  if (dtype == TS_F32)
    x.tile = rows <= 16 || brief ? AttnTile::k16 : AttnTile::k64;
  else
    x.tile = rows <= 16 ? AttnTile::k16 : rows <= 32 || brief || (rows <= 64 && pairs * 12 < cus) ? AttnTile::k32 : AttnTile::k128;
  x.rows = 16 << (int)x.tile;
  const bool small = x.tile == AttnTile::k16 || x.tile == AttnTile::k32;
  x.groups = cus * (c->head_dim == 256 ? 1 : x.tile == AttnTile::k16 && dtype == TS_BF16 && pairs >= cus ? 3 : 2);
  x.min_tokens = small ? 256 : 64;  // a step
  // Four steps of small tiles, six of tiles of 32 that have a compute unit each,
  // sixteen of large ones that fill the device, take less than cutting and joining:
  // nothing is cut (a tree of 65 rows over 1100 tokens: 17 us, cut 21; over 2000:
  // 23.5 and 23.6; one of 17 rows over 2000: 22 and 18; one row over 1100: 12.6 and
  // 12.9, over 2000 17 and 13).
  const int64_t tiles = (rows + x.rows - 1) / x.rows, all = tiles * c->heads * R;
  const int64_t uncut = x.tile == AttnTile::k32 && all <= cus ? 1536 : 1024;
  x.whole_tiles = tokens > 0 && tokens <= uncut && all < 1 << 24 && (small || all >= cus) ? (int)tiles : 0;
  // Few tiles are padded to whole pieces: a workgroup that ends one tile and begins
  // another pays for both (a tree of 65 rows over 5003 tokens, 72 tiles on 512
  // workgroups: 34.8 us, padded 29.7; three of 33 rows over 500 to 2500, 120 tiles:
  // 34 and 24). Padding costs up to a piece a tile, a quarter of all at the most.
  x.spare = !x.whole_tiles && all * 4 <= x.groups ? (int)all : 0;
  const size_t parts = (size_t)x.groups * 2 * x.rows;
  x.stats = parts * c->head_dim * sizeof(float);
  x.joins = x.stats + parts * sizeof(AttnStat);
  x.bytes = (x.joins + x.groups * sizeof(AttnJoin) + 255) & ~(size_t)255;
  if (x.whole_tiles) x.groups = (int)all;
  return x;
}

// Compute units of the current device (256 where there is none to ask).
int compute_units() {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      cus < 1) {
    (void)hipGetLastError();
    cus = 256;
  }
  return cus;
}

int64_t elem_size(int32_t dtype) { return dtype == TS_BF16 ? 2 : 4; }

}  // namespace
}  // namespace ts

using namespace ts;

#define TS_CHECK(call)                    \
  do {                                    \
    if (int32_t rc_ = (call)) return rc_; \
  } while (0)

extern "C" {

size_t ts_kv_block_bytes(int32_t page_size, int32_t head_dim) {
  if (!page_size_ok(page_size) || !head_dim_ok(head_dim)) return 0;
  return (size_t)page_size * head_dim * 17 / 16;
}

int32_t ts_kv_plan(const int32_t* len, const int32_t* n, int32_t R, int32_t cap, int32_t page_size,
                   int32_t num_pages, int32_t max_blocks, int32_t* free_pages, int32_t* free_count,
                   int32_t* held, int32_t* table, int32_t* slot, int32_t* granted, void* stream) {
  clear_error();
  if (!page_size_ok(page_size)) return fail(TS_EUNSUPPORTED, "page_size=%d is not 16, 32, 64, 128 or 256", page_size);
  TS_CHECK(check_requests(R, max_blocks, page_size));
  if (cap < 1 || cap > TS_KV_MAX_CAP) return fail(TS_EINVAL, "cap=%d outside [1, %d]", cap, TS_KV_MAX_CAP);
  if ((int64_t)R * cap >= (int64_t)1 << 31) return fail(TS_EUNSUPPORTED, "R * cap = %lld reaches 2^31", (long long)R * cap);
  if (num_pages < 1) return fail(TS_EINVAL, "num_pages=%d", num_pages);
  if ((int64_t)num_pages * page_size >= (int64_t)1 << 31)
    return fail(TS_EUNSUPPORTED, "num_pages * page_size = %lld reaches 2^31", (long long)num_pages * page_size);
  if ((int64_t)R * max_blocks + num_pages >= (int64_t)1 << 31)
    return fail(TS_EUNSUPPORTED, "R * max_blocks + num_pages = %lld reaches 2^31", (long long)R * max_blocks + num_pages);
  if (R == 0) return TS_OK;
  if (!len || !n || !free_pages || !free_count || !held || !table || !granted)
    return fail(TS_EINVAL, "a required array is NULL");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const KvPlanParams p = {len, n, R, cap, log2i(page_size), num_pages, max_blocks,
                          free_pages, free_count, held, table, slot, granted};
  launch_kv_plan(p, s);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

int32_t ts_kv_append(const ts_kv_cache* cache, int32_t layer, const void* k, const void* v, int32_t dtype,
                     int64_t k_stride, int64_t v_stride, const int32_t* slot, int32_t rows, void* stream) {
  clear_error();
  TS_CHECK(check_cache(cache));
  TS_CHECK(check_layer(cache, layer, 1));
  TS_CHECK(check_dtype(dtype));
  if (rows < 0) return fail(TS_EINVAL, "rows=%d is negative", rows);
  if (rows == 0) return TS_OK;
  if (!k || !v || !slot) return fail(TS_EINVAL, "k, v or slot is NULL");
  const int64_t width = (int64_t)cache->heads * cache->head_dim, unit = 16 / elem_size(dtype);
  if (k_stride < width || v_stride < width || k_stride % unit || v_stride % unit)
    return fail(TS_EINVAL, "strides %lld, %lld: at least %lld elements and whole 16 bytes are needed", (long long)k_stride,
                (long long)v_stride, (long long)width);
  if (!aligned16(k) || !aligned16(v)) return fail(TS_EINVAL, "k and v must start at 16-byte aligned addresses");
  if (rows * width > kMaxElements)
    return fail(TS_EUNSUPPORTED, "rows * heads * head_dim = %lld exceeds 2^34", (long long)(rows * width));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const KvAppendParams p = {view(cache, layer), k, v, k_stride, v_stride, slot, rows};
  launch_kv_append(p, cache->head_dim, dtype == TS_BF16, s);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

int32_t ts_kv_read(const ts_kv_cache* cache, int32_t layer, int32_t layers, const int32_t* slot, int32_t rows,
                   void* k, void* v, int32_t dtype, void* stream) {
  clear_error();
  TS_CHECK(check_cache(cache));
  TS_CHECK(check_layer(cache, layer, layers));
  TS_CHECK(check_dtype(dtype));
  if (rows < 0) return fail(TS_EINVAL, "rows=%d is negative", rows);
  if (rows == 0 || (!k && !v)) return TS_OK;
  if (!slot) return fail(TS_EINVAL, "slot is NULL");
  if (!aligned16(k) || !aligned16(v)) return fail(TS_EINVAL, "k and v must start at 16-byte aligned addresses");
  const int64_t width = (int64_t)cache->heads * cache->head_dim;
  if (rows * width > kMaxElements)
    return fail(TS_EUNSUPPORTED, "rows * heads * head_dim = %lld exceeds 2^34", (long long)(rows * width));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const KvReadParams p = {view(cache, layer), slot, rows, layers, k, v};
  launch_kv_read(p, cache->head_dim, dtype == TS_BF16, s);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

size_t ts_kv_attention_workspace_size(const ts_kv_cache* cache, int32_t R, int32_t cap, int32_t q_heads, int32_t dtype) {
  clear_error();
  if (check_cache(cache) || check_dtype(dtype) || R < 0 || R > kMaxRequests || cap < 1 || cap > TS_KV_MAX_CAP || q_heads < 1 ||
      q_heads % cache->heads || q_heads / cache->heads > kMaxGroup || (int64_t)R * cap * q_heads >= (int64_t)1 << 31)
    return 0;
  return attn_plan(cache, R, cap, q_heads, dtype, 0, compute_units()).bytes;
}

int32_t ts_kv_attention(const ts_kv_cache* cache, int32_t layer, const void* q, int32_t dtype, int64_t q_stride,
                        int32_t q_heads, const int32_t* len, const int32_t* n, int32_t R, int32_t cap,
                        const int32_t* table, int32_t max_blocks, const uint32_t* mask, float scale, void* out,
                        float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  TS_CHECK(check_cache(cache));
  TS_CHECK(check_layer(cache, layer, 1));
  TS_CHECK(check_dtype(dtype));
  TS_CHECK(check_requests(R, max_blocks, cache->page_size));
  if (q_heads < 1 || q_heads % cache->heads)
    return fail(TS_EINVAL, "q_heads=%d is no positive multiple of the cache's %d heads", q_heads, cache->heads);
  if (q_heads / cache->heads > kMaxGroup)
    return fail(TS_EUNSUPPORTED, "q_heads / heads = %d exceeds %d", q_heads / cache->heads, kMaxGroup);
  const int32_t most = mask ? TS_MAX_CAP : TS_KV_MAX_CAP;
  if (cap < 1 || cap > most) return fail(TS_EINVAL, "cap=%d outside [1, %d]", cap, most);
  if ((int64_t)R * cap * q_heads >= (int64_t)1 << 31)
    return fail(TS_EUNSUPPORTED, "R * cap * q_heads = %lld reaches 2^31", (long long)R * cap * q_heads);
  if (!std::isfinite(scale * kLog2e)) return fail(TS_EINVAL, "scale must be finite and below 2^127");
  if (R == 0) return TS_OK;
  if (!q || !len || !n || !table || !out) return fail(TS_EINVAL, "a required array is NULL");
  const int64_t width = (int64_t)q_heads * cache->head_dim;
  if (q_stride < width || q_stride % (16 / elem_size(dtype)))
    return fail(TS_EINVAL, "q_stride %lld: at least %lld elements and whole 16 bytes are needed", (long long)q_stride, (long long)width);
  if (!aligned16(q) || !aligned16(out)) return fail(TS_EINVAL, "q and out must start at 16-byte aligned addresses");
  const int cus = compute_units();
  const size_t need = attn_plan(cache, R, cap, q_heads, dtype, 0, cus).bytes;
  if (workspace_bytes < need) return fail(TS_ENOSPACE, "workspace %zu bytes < %zu needed", workspace_bytes, need);
  const AttnPlan plan = attn_plan(cache, R, cap, q_heads, dtype, (int64_t)max_blocks * cache->page_size, cus);
  if (!workspace || !aligned16(workspace)) return fail(TS_EINVAL, "workspace must be 16-byte aligned memory");
  if (q == out) return fail(TS_EINVAL, "out must not be the array q");
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const KvAttnParams p = {view(cache, layer), q, q_stride, q_heads, q_heads / cache->heads, R, cap, max_blocks,
                          ts_tree_mask_words(cap), len, n, table, mask, scale * kLog2e, out, lse, plan.min_tokens, plan.spare, plan.whole_tiles,
                          reinterpret_cast<float*>(ws), reinterpret_cast<AttnStat*>(ws + plan.stats),
                          reinterpret_cast<AttnJoin*>(ws + plan.joins)};
  const bool bf16 = dtype == TS_BF16;
  if (cache->head_dim == 64) launch_kv_attention_t<64>(p, plan.tile, bf16, plan.groups, s);
  if (cache->head_dim == 128) launch_kv_attention_t<128>(p, plan.tile, bf16, plan.groups, s);
  if (cache->head_dim == 256) launch_kv_attention_t<256>(p, plan.tile, bf16, plan.groups, s);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

int32_t ts_kv_accept(const ts_kv_cache* cache, const int32_t* len, const int32_t* n, int32_t R,
                     const int32_t* table, int32_t max_blocks, const int32_t* path_nodes,
                     const int32_t* path_len, int32_t* new_len, void* stream) {
  clear_error();
  TS_CHECK(check_cache(cache));
  TS_CHECK(check_requests(R, max_blocks, cache->page_size));
  if (R == 0) return TS_OK;
  if (!len || !n || !table || !path_nodes || !path_len || !new_len) return fail(TS_EINVAL, "a required array is NULL");
  if (new_len == len || new_len == n || new_len == table || new_len == path_nodes || new_len == path_len)
    return fail(TS_EINVAL, "new_len must not be one of the inputs");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const KvAcceptParams p = {view(cache, 0), cache->layers, len, n, table, path_nodes, path_len, R, max_blocks, new_len};
  launch_kv_accept(p, cache->head_dim, s);
  TS_HIP(hipGetLastError());
  return TS_OK;
}

}  // extern "C"
