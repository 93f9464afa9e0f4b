// Attention over the 8-bit cache: argument checks, workspace and choice of kernel.
#include <algorithm>
#include "kv_attend_host.hpp"

namespace glowq {

// Shares of a call's steps, and the fewest steps of one.  Few rows: a share to a compute unit, of any size (one request of 30000, 8
// heads: 19.5 us, 24 with 512); where units fill them anyway, shorter ones even out units of ragged lengths (64 requests up to
// 8000: 104 us, 109 with 256), but not below 16 steps (64 up to 1000: 19 us, 26 without that).
constexpr int FEW_SHARES = 256, FEW_FULL_SHARES = 768, FEW_FULL_LEAST = 16;
constexpr int MANY_SHARES = 512;       // (512 tokens on 8000: 84 us, 91 with 384, 101 with 768)
constexpr int MANY_LEAST = 8;          // fewer steps make more partial results (16 kB of a wave) than they save (4 x 30 new tokens on
                                       // 8000, 28 heads of 4: 40 us; 55 with 4, 42 with 16)
constexpr long long MOST_WORKGROUPS = 0xffffffffll / 256;       // a launch counts its threads in 32 bits
constexpr size_t KV_COUNT_BYTES = (3 * MANY_SHARES + 2 * FEW_FULL_SHARES) * 4;

// What a call launches, and where its partial results lie.
struct AttendPlan {
  int few, many;                       // workgroups
  int few_shares, few_least, many_shares;
  size_t off_many, off_few, bytes;
};

// Most keys of a request: no position or window below overflows 32 bits
static int longest(const glowq_kv_cache& c, const glowq_kv_query& p) {
  return (int)std::min<long long>(std::min<long long>((long long)p.table_width * c.block_tokens, p.max_length), 1 << 30);
}

// Workgroups that share the steps: never more than there can be, from the caller's bounds.  units: at most so many; least_rows: of
// a request that has any
static int plan_shares(const glowq_kv_cache& c, const glowq_kv_query& p, long long rows, int R, int step, int shares, long long* units,
                       int least_rows = 1) {
  const long long all = (long long)p.T * (p.heads / c.kv_heads), cap = longest(c, p);
  *units = c.kv_heads * std::min<long long>(p.n_requests * ((rows + R - 1) / R), all / R + std::min<long long>(p.n_requests, all / least_rows));
  const long long steps = (cap + 31 + step - 1) / step;
  return (int)std::min<long long>(shares, *units * steps);
}
static AttendPlan plan_attend(const glowq_kv_cache& c, const glowq_kv_query& p) {
  AttendPlan o = {};
  const long long rows = (long long)p.max_fresh * (p.heads / c.kv_heads);
  long long units;
  o.bytes = o.off_many = KV_COUNT_BYTES;
  const bool many = rows > KV_FEW_ROWS;
  if (many) {
    o.many_shares = plan_shares(c, p, rows, KV_MANY_ROWS, KV_MANY_STEP, MANY_SHARES, &units, p.n_requests > 1 ? KV_FEW_ROWS + 1 : 1);
    o.bytes += 3ull * o.many_shares * KV_MANY_ROWS * (c.head_dim + 2) * 4;
    o.many = o.many_shares ? (int)std::min<long long>(units + 2 * o.many_shares, 0x3fffffff) : 0;
  }
  o.off_few = o.bytes;
  if (!many || p.n_requests > 1) {     // (a single request's rows are taken as many, whatever they are)
    const int r = many ? KV_FEW_ROWS : (int)rows;
    o.few_shares = plan_shares(c, p, r, KV_FEW_ROWS, KV_FEW_STEP, FEW_SHARES, &units);
    o.few_least = 1;
    if (units >= FEW_SHARES) {
      o.few_shares = plan_shares(c, p, r, KV_FEW_ROWS, KV_FEW_STEP, FEW_FULL_SHARES, &units);
      o.few_least = FEW_FULL_LEAST;
    }
    o.bytes += 2ull * o.few_shares * KV_FEW_ROWS * (c.head_dim + 2) * 4;
    o.few = (int)std::min<long long>(units + o.few_shares, 0x3fffffff);
  }
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
  if ((long long)p->T * p->heads > 0x7fffffffll || (long long)p->n_requests * c->kv_heads > 0x7fffffffll) return GLOWQ_ERR_SHAPE;
  if (p->max_fresh < 1 || p->max_fresh > p->T || p->max_length < 1 || p->window < 0) return GLOWQ_ERR_SHAPE;
  if (!(p->scale > 0.f) || !(p->scale <= 3e38f)) return GLOWQ_ERR_SHAPE;
  if (p->act_dtype != GLOWQ_F16 && p->act_dtype != GLOWQ_BF16) return GLOWQ_ERR_DTYPE;
  const long long w = (long long)p->heads * c->head_dim;
  if (p->ldq < w || p->ldo < w) return GLOWQ_ERR_SHAPE;
  if (p->ldq % 8 || p->ldo % 8) return GLOWQ_ERR_UNSUPPORTED;
  const AttendPlan o = plan_attend(*c, *p);
  if ((long long)o.few + o.many > MOST_WORKGROUPS) return GLOWQ_ERR_SHAPE;
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
  a.cap = longest(c, p);
  a.window = p.window >= 1 << 30 ? 0 : p.window;       // (no key is so far behind another: longest)
  a.scale = p.scale * KV_LOG2E;
  KvCrew many = {o.few ? KV_FEW_ROWS : 0, 0x7fffffff, o.many_shares, MANY_LEAST, c.head_dim == 64 ? 3 * MANY_SHARES / 2 : MANY_SHARES, (uint32_t*)ws, (float*)(ws + o.off_many)};
  KvCrew few = {0, o.many ? KV_FEW_ROWS : 0x7fffffff, o.few_shares, o.few_least, 0, (uint32_t*)ws + 3 * MANY_SHARES, (float*)(ws + o.off_few)};
  return launch_kv_attend(a, many, few, o.many, o.few, p.act_dtype, st);
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
