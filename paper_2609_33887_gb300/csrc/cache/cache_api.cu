// The C entry points of libbdcache (bdcache.h): argument checks, workspaces,
// kernel choice. Checks come before any CUDA call.
#include <algorithm>
#include <climits>
#include <cmath>
#include <mutex>

#include "cache.h"
#include "host.h"
#include "trace.h"

extern "C" {

int bdkv_tables(const bdkv_tables_args* args, void* stream) {
  bd::TraceRange trace("bdkv_tables");
  if (args == nullptr) return BD_ERR_NULL;
  const bdkv_tables_args& a = *args;
  if (a.n_seq < 0 || a.n_seq > bdkv::MAX_SEQ_TABLES || !page_size_ok(a.page_size) || a.max_blocks < 0 ||
      a.max_tokens < 0 || a.table_stride < a.max_blocks || a.ring_size < 1 || a.ring_size > INT_MAX)
    return BD_ERR_SHAPE;
  if (!a.free_pages || !a.pool_in || !a.pool_out || !a.query_start ||
      (a.n_seq > 0 && (!a.lens || !a.new_tokens || !a.kv_lens || !a.status || (a.max_blocks > 0 && !a.block_table))) ||
      (a.max_tokens > 0 && (!a.slot_map || !a.positions)))
    return BD_ERR_NULL;
  if (a.pool_out == a.pool_in || (a.n_seq > 0 && a.kv_lens == a.lens)) return BD_ERR_ARG;
  if (!aligned(a.pool_in, 8) || !aligned(a.pool_out, 8) || !aligned(a.slot_map, 8) || !aligned(a.positions, 4) ||
      !aligned(a.lens, 4) || !aligned(a.new_tokens, 4) || !aligned(a.block_table, 4) || !aligned(a.free_pages, 4) ||
      !aligned(a.kv_lens, 4) || !aligned(a.query_start, 4) || !aligned(a.status, 4))
    return BD_ERR_ALIGN;
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  return cuda_status(bdkv::launch_tables(a, sms, static_cast<cudaStream_t>(stream)));
}

int bdkv_write(const bdkv_cache* cache, const bdkv_rows* k, const bdkv_rows* v, const int64_t* slot_map,
               int64_t n_tokens, void* stream) {
  bd::TraceRange trace("bdkv_write");
  if (!cache || !k || !v) return BD_ERR_NULL;
  if (int rc = check_cache(*cache)) return rc;
  if (int rc = check_rows(*k)) return rc;
  if (int rc = check_rows(*v)) return rc;
  if (k->dtype != v->dtype) return BD_ERR_DTYPE;
  if (int rc = check_cache_apart(*cache)) return rc;
  if (n_tokens < 0 || n_tokens > INT_MAX) return BD_ERR_SHAPE;
  if (n_tokens == 0) return BD_OK;
  if (!k->data || !v->data || !slot_map) return BD_ERR_NULL;
  if (!aligned(slot_map, 8)) return BD_ERR_ALIGN;
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  return cuda_status(
      bdkv::launch_write(*cache, *k, *v, slot_map, n_tokens, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

namespace {

int check_attention(const bdkv_cache* cache, const bdkv_attention_args* args) {
  if (!cache || !args) return BD_ERR_NULL;
  const bdkv_cache& c = *cache;
  const bdkv_attention_args& a = *args;
  if (int rc = check_cache(c)) return rc;
  if (int rc = check_rows(a.q)) return rc;
  if (int rc = check_rows(a.out)) return rc;
  if (a.out.dtype != a.q.dtype) return BD_ERR_DTYPE;
  if (a.n_seq < 0 || a.n_seq > 65535 || a.n_q_heads < 1 || a.n_q_heads % c.n_heads != 0 ||
      a.n_q_heads / c.n_heads > 64 || a.max_q_len < 0 || a.max_kv_len < 0 || a.max_kv_len > MAX_KV || a.max_blocks < 0 ||
      a.table_stride < a.max_blocks || a.table_stride > MAX_STRIDE ||
      a.max_kv_len > int64_t(a.max_blocks) * c.page_size ||
      int64_t(a.max_q_len) * (a.n_q_heads / c.n_heads) > (1 << 26))
    return BD_ERR_SHAPE;
  if (a.mask_block < 0 || !std::isfinite(a.scale)) return BD_ERR_ARG;
  if (a.n_seq > 0 && a.max_q_len > 0) {
    if (!a.q.data || !a.out.data || !a.kv_lens || !a.query_start || (a.max_blocks > 0 && !a.block_table))
      return BD_ERR_NULL;
    if (!aligned(a.kv_lens, 4) || !aligned(a.query_start, 4) || !aligned(a.block_table, 4) || !aligned(a.lse, 4) ||
        !aligned(a.workspace, 256))
      return BD_ERR_ALIGN;
    return check_rows_apart(a.out, a.n_q_heads, c.head_dim, a.n_seq > 1 || a.max_q_len > 1);
  }
  return BD_OK;
}

bdkv::AttnArgs attn_args(const bdkv_cache& c, const bdkv_attention_args& a) {
  bdkv::AttnArgs r = {};
  r.k = c.k, r.v = c.v, r.ks = c.k_scale, r.vs = c.v_scale;
  r.k_page = c.k_stride[0], r.k_tok = c.k_stride[1], r.k_head = c.k_stride[2];
  r.v_page = c.v_stride[0], r.v_tok = c.v_stride[1], r.v_head = c.v_stride[2];
  r.ks_page = c.k_scale_stride, r.vs_page = c.v_scale_stride;
  r.n_pages = c.n_pages;
  while ((1 << r.page_shift) < c.page_size) ++r.page_shift;
  r.dim = c.head_dim, r.n_kv = c.n_heads, r.group = a.n_q_heads / c.n_heads;
  r.q = a.q.data, r.q_tok = a.q.stride_token, r.q_head = a.q.stride_head;
  r.out = a.out.data, r.o_tok = a.out.stride_token, r.o_head = a.out.stride_head;
  r.lse = a.lse;
  r.table = a.block_table, r.table_stride = a.table_stride, r.max_blocks = a.max_blocks;
  r.kv_lens = a.kv_lens, r.q_start = a.query_start;
  r.n_seq = a.n_seq, r.max_q = a.max_q_len, r.max_kv = a.max_kv_len, r.mask_block = a.mask_block;
  r.coef = a.scale * bd::LOG2E;
  r.f16 = a.q.dtype == BDKV_F16;
  return r;
}

}  // namespace

namespace {

// How a call runs: the kernel, and its split along the cache.
struct Plan {
  bool tiles, one_tile, longest_first;
  int chunk, n_split;
  int64_t part_rows;  // rows of partial results
  size_t bytes;       // of workspace
};

// The kernel: up to 32 rows per key/value head (queries times the group) are one or two tiles of the row kernel (64
// requests of 300 to 4001 tokens, 4 heads: 20 rows 56 us, 60 in the tile kernel; 28 rows 56 and 61; 32 rows 57 and 51; 48
// rows 86 and 61. 8 requests, 8 heads: 32 rows 28 and 30).
// Two tiles of 128 rows to a CTA read the cache once for both; one where that still runs in one wave and the
// caches are too short to fill the device by a split (4 heads, 8 x 512 rows over 200 to 1400 tokens 21 us, 29 with two; 8
// heads, two waves of 32 x 256 rows over 700 to 4096 111 and 82; 2 x 256 rows over 20000 to 30000 84 and 71).
// The split along the cache. The host does not know how the lengths differ: one or two requests are split into one wave of
// CTAs (two to an SM for the row kernel, one for the other), more requests into finer parts, which even out. Row kernel:
// two caches of 131071 tokens 48 us in one wave, 69 in four; 16 requests of 57 to 60000 tokens 193 us in parts for 2 CTAs
// per SM, 159 for 3, 197 for 4. Tile kernel, parts of 2048 tokens or more (a part costs its rows' fp32 results): 2 x 64
// queries over 20000 to 30000 tokens 45 us in one wave, 61 in three; 8 x 9 queries over 300 to 30001 tokens 99 and 73.
// The parts follow the call's bound, not the lengths: one request of 1531 tokens takes 7.0 us under its own length, 14.1
// under a bound of 131072.
// More CTAs than run at once take the requests longest first: 64 requests x 35 rows over 300 to 4001 tokens 83 us in the
// requests' order and 60 so; 512 CTAs of equal lengths, where the order is for nothing, 261 and 262.
Plan make_plan(const bdkv_cache& c, const bdkv_attention_args& a, int sms) {
  Plan p = {};
  const int64_t rows = int64_t(a.max_q_len) * (a.n_q_heads / c.n_heads);
  p.tiles = rows > 2 * bdkv::ROWS_TILE;
  const int64_t pairs = int64_t(c.n_heads) * a.n_seq;
  const int64_t one_tile_ctas = (rows + bdkv::TILES_TILE - 1) / bdkv::TILES_TILE * pairs;
  p.one_tile = rows <= bdkv::TILES_TILE || (one_tile_ctas <= sms && a.max_kv_len <= 4096);
  const int64_t tile = !p.tiles ? bdkv::ROWS_TILE : p.one_tile ? bdkv::TILES_TILE : 2 * bdkv::TILES_TILE;
  const int64_t ctas = (rows + tile - 1) / tile * pairs;
  const bool few = a.n_seq <= 2;
  int64_t parts;
  if (p.tiles) {
    const int64_t finer = std::min<int64_t>((3 * int64_t(sms) + ctas - 1) / ctas, a.max_kv_len / 2048);
    parts = few || ctas >= sms ? sms / ctas : std::max<int64_t>(sms / ctas, finer);
  } else {
    parts = few ? 2 * int64_t(sms) / ctas : (3 * int64_t(sms) + ctas - 1) / ctas;
  }
  const int64_t least = p.tiles ? 256 : 128;  // tokens
  int64_t chunk = parts > 1 ? ((a.max_kv_len + parts - 1) / parts + 127) / 128 * 128 : a.max_kv_len;
  if (chunk < least) chunk = least;
  p.n_split = static_cast<int>((a.max_kv_len + chunk - 1) / chunk);
  p.longest_first = !few && a.n_seq <= bdkv::MAX_ORDERED && ctas * p.n_split > (p.tiles ? sms : 2 * sms);
  if (p.n_split <= 1) {
    p.n_split = 1;
    p.chunk = INT_MAX;
    return p;
  }
  p.chunk = static_cast<int>(chunk);
  p.part_rows = int64_t(a.n_seq) * a.max_q_len * a.n_q_heads * p.n_split;
  p.bytes = static_cast<size_t>(p.part_rows) * (c.head_dim + 1) * sizeof(float);
  return p;
}

}  // namespace

extern "C" {

size_t bdkv_attention_workspace(const bdkv_cache* cache, const bdkv_attention_args* args) {
  int sms = 0;
  if (check_attention(cache, args) != BD_OK || args->n_seq == 0 || args->max_q_len == 0 || check_device(&sms) != BD_OK)
    return 0;
  return make_plan(*cache, *args, sms).bytes;
}

int bdkv_attention(const bdkv_cache* cache, const bdkv_attention_args* args) {
  bd::TraceRange trace("bdkv_attention");
  if (int rc = check_attention(cache, args)) return rc;
  if (args->n_seq == 0 || args->max_q_len == 0) return BD_OK;
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  const cudaStream_t st = static_cast<cudaStream_t>(args->stream);
  const Plan plan = make_plan(*cache, *args, sms);
  bdkv::AttnArgs a = attn_args(*cache, *args);
  a.chunk = plan.chunk;
  a.n_split = plan.n_split;
  a.one_tile = plan.one_tile;
  a.longest_first = plan.longest_first;
  const auto run = [&](void* ws) {
    a.part_o = static_cast<float*>(ws);
    a.part_l = a.part_o + plan.part_rows * cache->head_dim;
    cudaError_t e = plan.tiles ? bdkv::launch_attn_tiles(a, st) : bdkv::launch_attn_rows(a, st);
    if (e == cudaSuccess && plan.n_split > 1) e = bdkv::launch_attn_join(a, st);
    return cuda_status(e);
  };
  if (plan.bytes == 0) return run(nullptr);
  if (args->workspace != nullptr) return args->workspace_bytes < plan.bytes ? BD_ERR_WORKSPACE : run(args->workspace);
  std::lock_guard<std::mutex> lock(g_mu);
  Workspace* w = nullptr;
  if (int rc = own_workspace(plan.bytes, st, &w)) return rc;
  const int rc = run(w->data);
  return cudaEventRecord(w->used, st) == cudaSuccess ? rc : BD_ERR_CUDA;
}

int bdkv_get_device_status(void* stream) {
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  uint32_t bits = 0;
  if (bdkv::tiles_status(static_cast<cudaStream_t>(stream), &bits) != cudaSuccess) return BD_ERR_CUDA;
  return bits ? BD_ERR_TIMEOUT : BD_OK;
}

int bdkv_shutdown(void) { return free_workspaces(); }

}  // extern "C"
