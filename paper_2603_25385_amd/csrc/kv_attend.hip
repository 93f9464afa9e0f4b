// Attention over the 8-bit cache: argument checks, workspace and choice of kernel.
#include <algorithm>
#include "kv_attend_host.hpp"

namespace glowq {

constexpr int FEW_PIECES = 1024;       // workgroups that few-row calls are cut into
constexpr int MANY_PIECES = 512;       // ... and calls of many rows
constexpr int FEW_ROWS = 32;           // most rows of a request that the few-row kernel serves

// What a call launches.
struct AttendPlan {
  bool few, many;
  int blocks;                          // of 16 rows in a tile of the few-row kernel
  int few_grid, many_grid;
  size_t bytes;
};
constexpr size_t KV_COUNT_BYTES = 2 * FEW_PIECES * 4;
static_assert(MANY_PIECES <= FEW_PIECES, "counts are sized for the larger number of pieces");

// Pieces are at most those wanted and one more for every tile, and no tile has more than its steps; slots are kept for tiles
// of two pieces and more, at most two for every piece wanted.
static int plan_kernel(const glowq_kv_cache& c, const glowq_kv_query& p, long long rows, long long cap, int R, int step, int pieces, size_t* bytes) {
  const long long all = (long long)p.T * (p.heads / c.kv_heads);
  const long long tiles = c.kv_heads * std::min<long long>(p.n_requests * ((rows + R - 1) / R), all / R + p.n_requests);
  const long long steps = (cap + 31 + step - 1) / step;
  const long long slots = std::min<long long>(2 * pieces, tiles * steps);
  *bytes = std::max(*bytes, KV_COUNT_BYTES + (size_t)slots * R * (c.head_dim + 2) * 4);
  return (int)std::min<long long>(std::min<long long>(pieces + tiles, tiles * steps), 0x7fffffff);
}
static AttendPlan plan_attend(const glowq_kv_cache& c, const glowq_kv_query& p) {
  AttendPlan o = {};
  const long long rows = (long long)p.max_fresh * (p.heads / c.kv_heads), cap = std::min<long long>((long long)p.table_width * c.block_tokens, p.max_length);
  o.many = rows > FEW_ROWS;
  o.few = !o.many || p.n_requests > 1;       // (a single request's rows are taken as many, whatever they are)
  o.blocks = rows <= 16 ? 1 : 2;
  if (o.few) o.few_grid = plan_kernel(c, p, o.many ? FEW_ROWS : rows, cap, 16 * o.blocks, 128, FEW_PIECES, &o.bytes);
  if (o.many) o.many_grid = plan_kernel(c, p, rows, cap, MANY_ROWS, 64, MANY_PIECES, &o.bytes);
  return o;
}

static bool bad16(const void* p) { return ((uintptr_t)p & 15u) != 0; }
static bool bad4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

static glowq_status check_query(const glowq_kv_cache* c, const glowq_kv_query* p, bool ptrs) {
  if (!c || !p) return GLOWQ_ERR_NULL;
  glowq_status s = kv_check_cache(c, ptrs);
  if (s != GLOWQ_OK) return s;
  if (p->n_requests < 1 || p->n_requests > (1 << 20) || p->T < 1 || p->T > (1 << 20) || p->table_width < 1) return GLOWQ_ERR_SHAPE;
  if (p->heads < 1 || p->heads > (1 << 12) || p->heads % c->kv_heads) return GLOWQ_ERR_SHAPE;
  if (p->max_fresh < 1 || p->max_fresh > p->T || p->max_length < 1 || p->window < 0) return GLOWQ_ERR_SHAPE;
  if (!(p->scale > 0.f) || !(p->scale <= 3e38f)) return GLOWQ_ERR_SHAPE;
  if (p->act_dtype != GLOWQ_F16 && p->act_dtype != GLOWQ_BF16) return GLOWQ_ERR_DTYPE;
  const long long w = (long long)p->heads * c->head_dim;
  if (p->ldq < w || p->ldo < w) return GLOWQ_ERR_SHAPE;
  if (p->ldq % 8 || p->ldo % 8) return GLOWQ_ERR_UNSUPPORTED;
  if (!ptrs) return GLOWQ_OK;
  if (!p->q || !p->out || !p->table || !p->lengths || !p->starts) return GLOWQ_ERR_NULL;
  return bad16(p->q) || bad16(p->out) || bad4(p->table) || bad4(p->lengths) || bad4(p->starts) ? GLOWQ_ERR_ALIGN : GLOWQ_OK;
}

static hipError_t launch_kv_attention(const glowq_kv_cache& c, const glowq_kv_query& p, char* ws, hipStream_t st) {
  const AttendPlan o = plan_attend(c, p);
  AttendArgs a;
  a.cache = kv_view(c);
  a.q = (const uint16_t*)p.q;
  a.out = (uint16_t*)p.out;
  a.table = p.table;
  a.lengths = p.lengths;
  a.starts = p.starts;
  a.ldq = p.ldq;
  a.ldo = p.ldo;
  a.width = p.table_width;
  a.n = p.n_requests;
  a.T = p.T;
  a.heads = p.heads;
  a.group = p.heads / c.kv_heads;
  a.max_fresh = p.max_fresh;
  a.cap = (int)std::min<long long>((long long)p.table_width * c.block_tokens, p.max_length);
  a.window = p.window;
  a.scale = p.scale * KV_LOG2E;
  a.counts = (uint32_t*)ws;
  a.slots = (float*)(ws + KV_COUNT_BYTES);
  a.least = 1;
  a.rows_from = 0;
  a.rows_to = o.many ? FEW_ROWS : 0x7fffffff;
  a.pieces = FEW_PIECES;
  if (o.few) {
    const hipError_t e = launch_kv_attend_few(a, p.act_dtype, o.blocks, o.few_grid, st);
    if (e != hipSuccess || !o.many) return e;
    a.rows_from = FEW_ROWS;
  }
  a.rows_to = 0x7fffffff;
  a.pieces = MANY_PIECES;
  return launch_kv_attend_many(a, p.act_dtype, o.many_grid, st);
}

}  // namespace glowq

using namespace glowq;
extern "C" {

glowq_status glowq_kv_attention_workspace_bytes(const glowq_kv_cache* cache, const glowq_kv_query* query, size_t* bytes) {
  if (!bytes) return GLOWQ_ERR_NULL;
  const glowq_status s = check_query(cache, query, false);
  if (s != GLOWQ_OK) return s;
  *bytes = plan_attend(*cache, *query).bytes;
  return GLOWQ_OK;
}

glowq_status glowq_kv_attention(const glowq_kv_cache* cache, const glowq_kv_query* query, void* workspace, size_t workspace_bytes, void* stream) {
  const glowq_status s = check_query(cache, query, true);
  if (s != GLOWQ_OK) return s;
  if (!workspace || workspace_bytes < plan_attend(*cache, *query).bytes) return GLOWQ_ERR_WORKSPACE;
  if ((uintptr_t)workspace & 255u) return GLOWQ_ERR_ALIGN;
  return hip_status(launch_kv_attention(*cache, *query, (char*)workspace, (hipStream_t)stream));
}

}  // extern "C"
