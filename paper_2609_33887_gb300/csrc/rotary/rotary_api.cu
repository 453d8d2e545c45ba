// The C entry points of libbdrotary (bdrotary.h): argument checks, tensor maps,
// workspaces, the split of an attention. Checks come before any CUDA call.
#include <cmath>
#include <cudaTypedefs.h>

#include "cache/host.h"
#include "rotary/latent.h"
#include "trace.h"

namespace {

constexpr double MIN_SCALE = 0x1p-96;  // below it the sines' factor, scale * 2 pi / 2^32, leaves fp32's normal numbers
constexpr int64_t MAX_TMA_STRIDE = int64_t(1) << 38;  // elements of 16 bits: below 2^40 bytes

int check_rotary(const bdrot_rotary& r, int64_t head_dim) {
  if (r.dim < 16 || r.dim > 256 || r.dim % 16 != 0 || r.dim > head_dim) return BD_ERR_SHAPE;
  if ((r.interleaved != 0 && r.interleaved != 1) || !std::isfinite(static_cast<float>(r.scale)))
    return BD_ERR_ARG;
  if (r.scale != 0 && std::fabs(r.scale) < MIN_SCALE) return BD_ERR_ARG;
  if (!r.turns) return BD_ERR_NULL;
  return aligned(r.turns, 16) ? BD_OK : BD_ERR_ALIGN;
}

bdrot::Turn turn_of(const bdrot_rotary& r, const int32_t* positions, bool back) {
  bdrot::Turn t = {};
  t.turns = reinterpret_cast<const unsigned long long*>(r.turns);
  t.positions = positions;
  t.dim = r.dim, t.inter = r.interleaved != 0, t.back = back;
  const double radians = 1.4629180792671596e-9 * r.scale;  // 2 pi / 2^32
  t.scale = static_cast<float>(r.scale), t.scale_low = static_cast<float>(r.scale - t.scale);
  t.radians = static_cast<float>(radians), t.radians_low = static_cast<float>(radians - t.radians);
  return t;
}

// Whether rows a [n, heads_a, dim_a] and b [n, heads_b, dim_b] share memory: exact where they have the same strides (those of
// one token, or of one head on either side, aside), else whether their address ranges meet.
bool rows_meet(const bdkv_rows& a, int64_t heads_a, int64_t dim_a, const bdkv_rows& b, int64_t heads_b, int64_t dim_b,
               int64_t n) {
  using wide = __int128;
  const wide delta = (static_cast<wide>(reinterpret_cast<uintptr_t>(b.data)) -
                      static_cast<wide>(reinterpret_cast<uintptr_t>(a.data))) / 2;
  const auto span = [&](const bdkv_rows& r, int64_t heads, int64_t dim) {
    return static_cast<wide>(n - 1) * r.stride_token + static_cast<wide>(heads - 1) * r.stride_head + dim;
  };
  if (delta >= span(a, heads_a, dim_a) || -delta >= span(b, heads_b, dim_b)) return false;
  const int64_t t = a.stride_token, h = heads_a > 1 ? a.stride_head : b.stride_head;  // (of a single head it says nothing)
  if ((n > 1 && t != b.stride_token) || (heads_a > 1 && heads_b > 1 && h != b.stride_head)) return true;
  const auto floor_div = [](wide x, wide d) { return x >= 0 ? x / d : -((-x + d - 1) / d); };
  for (int64_t d = 1 - heads_a; d < heads_b; ++d) {  // a head of b less one of a, and k tokens: -dim_b < x + k t < dim_a?
    const wide x = delta + static_cast<wide>(d) * h;
    wide lo = 0, hi = 0;
    if (n > 1 && t > 0) {
      lo = std::max<wide>(-floor_div(x + dim_b - 1, t), 1 - n);
      hi = std::min<wide>(floor_div(dim_a - 1 - x, t), n - 1);
      if (lo <= hi) return true;
    } else if (x < dim_a && x > -dim_b) {
      return true;
    }
  }
  return false;
}

bool same_rows(const bdkv_rows& a, const bdkv_rows& b, int64_t heads, int64_t n) {
  return a.data == b.data && (n <= 1 || a.stride_token == b.stride_token) && (heads <= 1 || a.stride_head == b.stride_head);
}

// Rows that are turned into `out`, for n > 0 tokens.
int check_turned(const bdkv_rows& x, const bdkv_rows& out, int64_t heads, int64_t head_dim, int64_t n) {
  if (int rc = check_rows(x)) return rc;
  if (int rc = check_rows(out)) return rc;
  if (x.dtype != out.dtype) return BD_ERR_DTYPE;
  if (n == 0) return BD_OK;
  if (!x.data || !out.data) return BD_ERR_NULL;
  if (int rc = check_rows_apart(out, heads, head_dim, n > 1)) return rc;
  if (heads > 1 && n > 1 && out.stride_head > out.stride_token &&
      out.stride_head < static_cast<__int128>(n - 1) * out.stride_token + head_dim)
    return BD_ERR_ARG;  // a head's tokens reach into the next head's
  return same_rows(x, out, heads, n) || !rows_meet(x, heads, head_dim, out, heads, head_dim, n) ? BD_OK : BD_ERR_ARG;
}

int check_latent(const bdrot_latent& c) {
  if (!page_size_ok(c.page_size) || c.latent_dim < 16 || c.latent_dim > 512 || c.latent_dim % 16 != 0 || c.rope_dim < 16 ||
      c.rope_dim > 64 || c.rope_dim % 16 != 0 || c.n_pages < 0 || c.n_pages > INT_MAX)
    return BD_ERR_SHAPE;
  if (c.dtype != BDKV_BF16 && c.dtype != BDKV_F16) return BD_ERR_DTYPE;
  for (const int64_t* s : {c.latent_stride, c.rope_stride}) {
    if (int rc = check_strides(s, 2, 8)) return rc;
    if (s[0] >= MAX_TMA_STRIDE || s[1] >= MAX_TMA_STRIDE) return BD_ERR_SHAPE;
  }
  if (c.n_pages > 0 && (!c.latent || !c.rope)) return BD_ERR_NULL;
  if (!aligned(c.latent, 16) || !aligned(c.rope, 16)) return BD_ERR_ALIGN;
  // tokens that lie on one another
  const struct { const int64_t* s; int64_t dim; } parts[2] = {{c.latent_stride, c.latent_dim}, {c.rope_stride, c.rope_dim}};
  for (const auto& p : parts) {
    const int64_t page = p.s[0], tok = p.s[1], pages = c.n_pages;
    if (tok < p.dim) return BD_ERR_ARG;
    if (pages <= 1) continue;
    if (page >= tok ? static_cast<__int128>(page) < static_cast<__int128>(tok) * (c.page_size - 1) + p.dim
                    : page < p.dim || static_cast<__int128>(tok) < static_cast<__int128>(page) * (pages - 1) + p.dim)
      return BD_ERR_ARG;
  }
  return BD_OK;
}

// Latents and key parts of a cache that is written must not lie on one another either.
int check_latent_apart(const bdrot_latent& c) {
  if (c.n_pages == 0) return BD_OK;
  const bdkv_rows l = {c.latent, c.dtype, c.latent_stride[0], c.latent_stride[1]};  // a page's tokens as a row's heads
  const bdkv_rows r = {c.rope, c.dtype, c.rope_stride[0], c.rope_stride[1]};
  return rows_meet(l, c.page_size, c.latent_dim, r, c.page_size, c.rope_dim, c.n_pages) ? BD_ERR_ARG : BD_OK;
}

int check_attention(const bdrot_latent* cache, const bdrot_latent_attention_args* args) {
  if (!cache || !args) return BD_ERR_NULL;
  const bdrot_latent& c = *cache;
  const bdrot_latent_attention_args& a = *args;
  if (int rc = check_latent(c)) return rc;
  if (int rc = check_rows(a.q)) return rc;
  if (int rc = check_rows(a.out)) return rc;
  if (a.out.dtype != a.q.dtype || a.q.dtype != c.dtype) return BD_ERR_DTYPE;
  if (a.n_seq < 0 || a.n_seq > 65535 || a.n_heads < 1 || a.n_heads > 1024 || a.max_q_len < 0 || a.max_kv_len < 0 ||
      a.max_kv_len > MAX_KV || a.max_blocks < 0 || a.table_stride < a.max_blocks || a.table_stride > MAX_STRIDE ||
      a.max_kv_len > int64_t(a.max_blocks) * c.page_size || int64_t(a.max_q_len) * a.n_heads > (1 << 26))
    return BD_ERR_SHAPE;
  if (a.mask_block < 0 || !std::isfinite(a.scale * bd::LOG2E)) return BD_ERR_ARG;
  if (a.n_seq == 0 || a.max_q_len == 0) return BD_OK;
  if (!a.q.data || !a.out.data || !a.kv_lens || !a.query_start || (a.max_blocks > 0 && !a.block_table)) return BD_ERR_NULL;
  if (!aligned(a.kv_lens, 4) || !aligned(a.query_start, 4) || !aligned(a.block_table, 4) || !aligned(a.lse, 4) ||
      !aligned(a.workspace, 256))
    return BD_ERR_ALIGN;
  return check_rows_apart(a.out, a.n_heads, c.latent_dim, a.n_seq > 1 || a.max_q_len > 1);
}

// How a call's work is shared out.
struct Plan {
  int rows, row_tiles;
  bool shared, longest_first;
  int64_t part_rows;  // rows of partial results, two units to each CTA
  size_t bytes;       // of workspace: those, with a reference and a sum each, and two words for each unit
};

// Up to one unit for each SM the CTAs add up the tiles of all units, of lengths that the host does not know, and take equal
// shares of them, or a unit each where that is as good (64 units of 57 to 8189 tokens 66 us, a unit each 134, in parts of
// equal lengths, two to an SM, 75). With more units a CTA to each, the longest requests first (320 units of 300 to 4001
// tokens 125 us; in shares, whose CTAs change units more often and read less of what others read at the same time, 165 when
// this took 129).
Plan make_plan(const bdrot_latent& c, const bdrot_latent_attention_args& a, int sms) {
  Plan p = {};
  const int64_t rows = int64_t(a.max_q_len) * a.n_heads;
  p.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  p.row_tiles = static_cast<int>((rows + p.rows - 1) / p.rows);
  const int64_t units = int64_t(p.row_tiles) * a.n_seq, tiles = a.max_kv_len / bdrot::TOKENS + 1;
  p.shared = units <= std::min(sms, bdrot::MAX_SHARED_UNITS) && units * tiles < (int64_t(1) << 30);
  p.longest_first = !p.shared && a.n_seq > 2 && a.n_seq <= bdkv::MAX_ORDERED && units > sms;
  if (!p.shared) return p;
  p.part_rows = 2 * int64_t(sms) * p.rows;
  p.bytes = static_cast<size_t>(p.part_rows) * (c.latent_dim + 2) * sizeof(float) + static_cast<size_t>(units + 1) * 8;
  return p;
}

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> known{nullptr};
  if (auto f = known.load(std::memory_order_acquire)) return f;
  cudaDriverEntryPointQueryResult q;
  void* fn = nullptr;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
      q != cudaDriverEntryPointSuccess)
    return nullptr;
  known.store(reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn), std::memory_order_release);
  return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
}

// Boxes of 64 elements by a page's tokens (or a tile's, of larger pages), or of as many columns of 64 elements as a stage of
// the attention kernel holds, by a tile's tokens. A cache without pages gets a map of one page over `any`, which no box
// reads: page numbers outside the cache are taken to the coordinate behind its last page.
bool encode(CUtensorMap* m, const bdrot_latent& c, const void* data, const int64_t* stride, int dim, int columns,
            const void* any) {
  const auto f = encoder();
  if (f == nullptr) return false;
  const cuuint64_t tok = (c.n_pages > 0 ? stride[1] : dim) * 2, page = c.n_pages > 1 ? stride[0] * 2 : tok;  // (one page's stride says nothing)
  const cuuint64_t tokens = c.page_size, pages = std::max<int64_t>(c.n_pages, 1);
  const cuuint64_t dims[2][4] = {{static_cast<cuuint64_t>(dim), tokens, pages}, {64, tokens, static_cast<cuuint64_t>(dim / 64), pages}};
  const cuuint64_t strides[2][3] = {{tok, page}, {tok, 128, page}};
  const cuuint32_t most = std::min(c.page_size, bdrot::TOKENS);
  const cuuint32_t box[2][4] = {{64, most, 1}, {64, most, static_cast<cuuint32_t>(columns), 1}}, step[4] = {1, 1, 1, 1};
  const int kind = columns > 0;
  return f(m, c.dtype == BDKV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3 + kind,
           const_cast<void*>(c.n_pages > 0 ? data : any), dims[kind], strides[kind], box[kind], step,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bdrot::LatentArgs latent_args(const bdrot_latent& c, const bdrot_latent_attention_args& a, const Plan& plan) {
  bdrot::LatentArgs p = {};
  bdkv::AttnArgs& r = p.a;
  r.n_pages = c.n_pages;
  while ((1 << r.page_shift) < c.page_size) ++r.page_shift;
  r.dim = c.latent_dim, r.n_kv = 1, r.group = a.n_heads;
  p.rope_dim = c.rope_dim, p.rows = plan.rows, p.row_tiles = plan.row_tiles, p.shared = plan.shared;
  r.q = a.q.data, r.q_tok = a.q.stride_token, r.q_head = a.q.stride_head;
  r.out = a.out.data, r.o_tok = a.out.stride_token, r.o_head = a.out.stride_head;
  r.lse = a.lse;
  r.table = a.block_table, r.table_stride = a.table_stride, r.max_blocks = a.max_blocks;
  r.kv_lens = a.kv_lens, r.q_start = a.query_start;
  r.n_seq = a.n_seq, r.max_q = a.max_q_len, r.max_kv = a.max_kv_len, r.mask_block = a.mask_block;
  r.coef = a.scale * bd::LOG2E;
  r.f16 = a.q.dtype == BDKV_F16;
  r.longest_first = plan.longest_first;
  return p;
}

}  // namespace

extern "C" {

int bdrot_rotate(const bdrot_rotary* rotary, const bdkv_rows* x, const bdkv_rows* out, int32_t n_heads,
                 int32_t head_dim, const int32_t* positions, int64_t n_tokens, int32_t inverse, void* stream) {
  bd::TraceRange trace("bdrot_rotate");
  if (!rotary || !x || !out) return BD_ERR_NULL;
  if (n_heads < 1 || n_heads > 1024 || head_dim < 16 || head_dim > 1024 || head_dim % 16 != 0 || n_tokens < 0 ||
      n_tokens > INT_MAX)
    return BD_ERR_SHAPE;
  if (inverse != 0 && inverse != 1) return BD_ERR_ARG;
  if (int rc = check_rotary(*rotary, head_dim)) return rc;
  if (int rc = check_turned(*x, *out, n_heads, head_dim, n_tokens)) return rc;
  if (n_tokens == 0) return BD_OK;
  if (!positions) return BD_ERR_NULL;
  if (!aligned(positions, 4)) return BD_ERR_ALIGN;
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  int64_t blocks = 0;
  const bdrot::RotateArgs a =
      bdrot::rotate_args(*x, *out, n_heads, head_dim, turn_of(*rotary, positions, inverse != 0), n_tokens, sms, &blocks);
  return cuda_status(bdrot::launch_rotate(a, blocks, x->dtype == BDKV_F16, static_cast<cudaStream_t>(stream)));
}

int bdrot_write(const bdrot_rotary* rotary, const bdkv_cache* cache, const bdkv_rows* k, const bdkv_rows* v,
                const int64_t* slot_map, const int32_t* positions, int64_t n_tokens, const bdkv_rows* q,
                const bdkv_rows* q_out, int32_t n_q_heads, void* stream) {
  bd::TraceRange trace("bdrot_write");
  if (!rotary || !cache || !k || !v || !q != !q_out) return BD_ERR_NULL;
  if (int rc = check_cache(*cache)) return rc;
  if (int rc = check_rows(*k)) return rc;
  if (int rc = check_rows(*v)) return rc;
  if (k->dtype != v->dtype || (q && q->dtype != k->dtype)) return BD_ERR_DTYPE;
  if (int rc = check_cache_apart(*cache)) return rc;
  if (int rc = check_rotary(*rotary, cache->head_dim)) return rc;
  if (n_tokens < 0 || n_tokens > INT_MAX || (q && (n_q_heads < 1 || n_q_heads > 1024))) return BD_ERR_SHAPE;
  if (q)
    if (int rc = check_turned(*q, *q_out, n_q_heads, cache->head_dim, n_tokens)) return rc;
  if (n_tokens == 0) return BD_OK;
  if (!k->data || !v->data || !slot_map || !positions) return BD_ERR_NULL;
  if (!aligned(slot_map, 8) || !aligned(positions, 4)) return BD_ERR_ALIGN;
  if (q)
    for (const bdkv_rows* r : {k, v})
      if (rows_meet(*r, cache->n_heads, cache->head_dim, *q_out, n_q_heads, cache->head_dim, n_tokens)) return BD_ERR_ARG;
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  const bdrot::Turn turn = turn_of(*rotary, positions, false);
  bdrot::RotateArgs turned = {};
  int64_t blocks = 0;
  if (q) turned = bdrot::rotate_args(*q, *q_out, n_q_heads, cache->head_dim, turn, n_tokens, sms, &blocks);
  return cuda_status(bdrot::launch_write(*cache, *k, *v, slot_map, n_tokens, turn, q ? &turned : nullptr, blocks, sms,
                                         static_cast<cudaStream_t>(stream)));
}

int bdrot_latent_write(const bdrot_rotary* rotary, const bdrot_latent* cache, const bdkv_rows* latent,
                       const bdkv_rows* rope, const int64_t* slot_map, const int32_t* positions, int64_t n_tokens,
                       void* stream) {
  bd::TraceRange trace("bdrot_latent_write");
  if (!cache || !latent || !rope) return BD_ERR_NULL;
  if (int rc = check_latent(*cache)) return rc;
  for (const bdkv_rows* r : {latent, rope}) {
    bdkv_rows one = *r;
    one.stride_head = 0;
    if (int rc = check_rows(one)) return rc;
    if (r->dtype != cache->dtype) return BD_ERR_DTYPE;
  }
  if (int rc = check_latent_apart(*cache)) return rc;
  if (rotary) {
    if (int rc = check_rotary(*rotary, cache->rope_dim)) return rc;
    if (rotary->dim != cache->rope_dim) return BD_ERR_SHAPE;
  }
  if (n_tokens < 0 || n_tokens > INT_MAX) return BD_ERR_SHAPE;
  if (n_tokens == 0) return BD_OK;
  if (!latent->data || !rope->data || !slot_map || (rotary && !positions)) return BD_ERR_NULL;
  if (!aligned(slot_map, 8) || (rotary && !aligned(positions, 4))) return BD_ERR_ALIGN;
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  bdrot::Turn turn = {};
  if (rotary) turn = turn_of(*rotary, positions, false);
  return cuda_status(bdrot::launch_latent_write(*cache, *latent, *rope, slot_map, n_tokens, rotary ? &turn : nullptr,
                                                sms, static_cast<cudaStream_t>(stream)));
}

size_t bdrot_latent_attention_workspace(const bdrot_latent* cache, const bdrot_latent_attention_args* args) {
  int sms = 0;
  if (check_attention(cache, args) != BD_OK || args->n_seq == 0 || args->max_q_len == 0 || check_device(&sms) != BD_OK)
    return 0;
  return make_plan(*cache, *args, sms).bytes;
}

int bdrot_latent_attention(const bdrot_latent* cache, const bdrot_latent_attention_args* args) {
  bd::TraceRange trace("bdrot_latent_attention");
  if (int rc = check_attention(cache, args)) return rc;
  if (args->n_seq == 0 || args->max_q_len == 0) return BD_OK;
  // (of the first token: how many there are is on the device)
  if (rows_meet(args->q, args->n_heads, cache->latent_dim + cache->rope_dim, args->out, args->n_heads, cache->latent_dim, 1))
    return BD_ERR_ARG;
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  const cudaStream_t st = static_cast<cudaStream_t>(args->stream);
  const Plan plan = make_plan(*cache, *args, sms);
  bdrot::LatentArgs p = latent_args(*cache, *args, plan);
  CUtensorMap latent, rope;
  p.columns = cache->page_size >= bdrot::TOKENS && cache->latent_dim % 64 == 0;
  const int columns = p.columns ? 2 * bdrot::pairs_per_stage((cache->latent_dim + 127) / 128) : 0;
  if (!encode(&latent, *cache, cache->latent, cache->latent_stride, cache->latent_dim, columns, args->q.data) ||
      !encode(&rope, *cache, cache->rope, cache->rope_stride, cache->rope_dim, 0, args->q.data))
    return BD_ERR_CUDA;
  const auto run = [&](void* ws) {
    p.a.part_o = static_cast<float*>(ws);
    p.a.part_l = p.a.part_o + plan.part_rows * cache->latent_dim;
    p.plan = reinterpret_cast<int2*>(p.a.part_l + plan.part_rows * 2);
    cudaError_t e = bdrot::launch_latent_attn(p, latent, rope, sms, st);
    if (e == cudaSuccess && plan.shared) e = bdrot::launch_latent_join(p, sms, st);
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

int bdrot_get_device_status(void* stream) {
  int sms = 0;
  if (int rc = check_device(&sms)) return rc;
  uint32_t bits = 0;
  if (bdrot::latent_status(static_cast<cudaStream_t>(stream), &bits) != cudaSuccess) return BD_ERR_CUDA;
  return bits ? BD_ERR_TIMEOUT : BD_OK;
}

int bdrot_shutdown(void) { return free_workspaces(); }

}  // extern "C"
