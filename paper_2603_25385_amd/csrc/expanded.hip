// Attention over rows of keys and values (latent attention, expanded): argument checks, workspace, launch.
#include <algorithm>
#include "attend_join.hpp"
#include "expanded.hpp"
#include "launch.hpp"

namespace glowq {

// (Heads of 128 + 64: 80 KB of LDS, two workgroups on a CU.)
template <int ACT, int N, int ROPE>
__global__ void __launch_bounds__(EXPANDED_THREADS, 2) k_expanded(ExpandedArgs x, KvCrew crew, JoinTicket* tickets, int slots) {
  __shared__ ExpandedLds<N, ROPE> lds;
  KvRequest req;
  long long all, total;
  const KvPart pc = kv_cut<EXPANDED_ROWS, EXPANDED_STEP>(x.a, crew, blockIdx.x, req, all, total);
  if (tickets) join_leave(tickets, slots, pc, req);
  if (pc.r >= 0) expanded_part<ACT, N, ROPE>(x, crew, pc, req, lds);
}

template <int ACT, int N>
__global__ void __launch_bounds__(JOIN_THREADS) k_expanded_join(ExpandedArgs x, KvCrew crew, const JoinTicket* tickets) {
  __shared__ float scratch[JOIN_THREADS][6];
  constexpr int R = EXPANDED_ROWS;
  const AttendArgs& a = x.a;
  KvRequest req;
  KvPart pc;
  if (!join_take(tickets, pc, req)) return;
  expanded_keys(x, pc.r, req);
  const int row0 = pc.tile * R, rows = min(R, req.rows - row0);
  attend_join<R, N>(crew, pc, rows, (rows + 31) / 32 * (32 * N / 4), scratch,
    [](int item, int& row, int& dim) {
      row = item / (64 * (N / 32) * 4) * 32 + (item & 31);
      dim = item / 64 % (N / 32 * 4) * 8 + (item >> 5 & 1) * 4;
    },
    [&](float l, int row) { return expanded_inverse(l, req, row0 + row); },
    [&](int row, int dim, float4_t v) {
      typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
      *(u32x2_t*)(a.out + (size_t)(req.start + row0 + row) * a.ldo + (size_t)pc.head * N + dim) = u32x2_t{kv_pack<ACT>(v[0], v[1]), kv_pack<ACT>(v[2], v[3])};
    });
}

// Shares: as many as the machine holds workgroups of heads of 128; steps of a part at least.  With 256, 512, 768 shares: pieces of three prompts on 16000
// 120, 130, 125 us, the long prompt 615 to 622, ragged prompts 47 to 48 each.  With 4, 8, 16 steps: the pieces 130 each, two pieces of up to 64 on 6000
// 32.5, 32.8, 33.9.
constexpr int EXPANDED_SHARES = 512, EXPANDED_LEAST = 8;
constexpr long long MOST_WORKGROUPS = 0xffffffffll / EXPANDED_THREADS;       // a launch counts its threads in 32 bits
constexpr int MOST_STRIDE = 1 << 24;       // a tile's offsets stay inside 32 bits

struct ExpandedPlan {
  int shares, workgroups;
  int slots;                   // partial results, at most: parts of units that are cut are fewer than two for every share
  bool cut;                    // whether a unit can be
  size_t bytes;
};

static int longest(const glowq_expanded_query& p) { return std::min(std::min(p.keys, p.max_length), 1 << 30); }

static ExpandedPlan plan_expanded(const glowq_expanded_query& p) {
  ExpandedPlan o = {};
  const int R = EXPANDED_ROWS;
  const long long units = p.heads * std::min<long long>(p.n_requests * (((long long)p.max_fresh + R - 1) / R), p.T / R + std::min<long long>(p.n_requests, p.T));
  const long long steps = (longest(p) + EXPANDED_STEP - 1) / EXPANDED_STEP;
  o.shares = (int)std::min<long long>(EXPANDED_SHARES, units * steps);
  o.cut = steps > EXPANDED_LEAST;
  o.workgroups = (int)std::min<long long>(units + (o.cut ? o.shares : 0), 0x3fffffff);
  o.slots = o.cut ? std::min(o.workgroups, 2 * o.shares) : 0;
  o.bytes = std::max<size_t>((size_t)o.slots * (R * (p.v_dim + 2) * 4 + sizeof(JoinTicket)), 256);
  return o;
}

static bool bad16(const void* p) { return ((uintptr_t)p & 15u) != 0; }
static bool bad4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

static glowq_status check_query(const glowq_expanded_query* p, bool ptrs) {
  if (!p) return GLOWQ_ERR_NULL;
  if (p->n_requests < 1 || p->n_requests > (1 << 20) || p->T < 1 || p->T > (1 << 20) || p->keys < 1 || p->keys > (1 << 30)) return GLOWQ_ERR_SHAPE;
  if (p->heads < 1 || p->heads > 1024 || p->nope_dim < 1 || p->rope_dim < 1 || p->v_dim < 1) return GLOWQ_ERR_SHAPE;
  if (p->max_fresh < 1 || p->max_fresh > p->T || p->max_length < 1) return GLOWQ_ERR_SHAPE;
  if (!(p->scale > 0.f) || !(p->scale <= 2e38f)) return GLOWQ_ERR_SHAPE;
  if ((p->nope_dim != 64 && p->nope_dim != 128) || p->v_dim != p->nope_dim || (p->rope_dim != 32 && p->rope_dim != 64)) return GLOWQ_ERR_UNSUPPORTED;
  if (p->act_dtype != GLOWQ_F16 && p->act_dtype != GLOWQ_BF16) return GLOWQ_ERR_DTYPE;
  const long long h = p->heads - 1;
  if (p->lhq < p->nope_dim + p->rope_dim || p->lhk < p->nope_dim || p->lhv < p->v_dim) return GLOWQ_ERR_SHAPE;
  if (h * p->lhq + p->nope_dim + p->rope_dim > p->ldq || h * p->lhk + p->nope_dim > p->ldk || h * p->lhv + p->v_dim > p->ldv ||
      p->ldr < p->rope_dim || p->ldo < p->heads * p->v_dim) return GLOWQ_ERR_SHAPE;
  if (p->ldk > MOST_STRIDE || p->ldv > MOST_STRIDE || p->ldr > MOST_STRIDE) return GLOWQ_ERR_SHAPE;
  if (p->ldq % 8 || p->lhq % 8 || p->ldk % 8 || p->lhk % 8 || p->ldr % 8 || p->ldv % 8 || p->lhv % 8 || p->ldo % 8) return GLOWQ_ERR_UNSUPPORTED;
  if (plan_expanded(*p).workgroups > MOST_WORKGROUPS) return GLOWQ_ERR_SHAPE;
  if (!ptrs) return GLOWQ_OK;
  if (!p->q || !p->k || !p->k_rope || !p->v || !p->out || !p->starts || !p->key_starts || !p->lengths) return GLOWQ_ERR_NULL;
  return bad16(p->q) || bad16(p->k) || bad16(p->k_rope) || bad16(p->v) || bad16(p->out) || bad4(p->starts) || bad4(p->key_starts) || bad4(p->lengths)
             ? GLOWQ_ERR_ALIGN : GLOWQ_OK;
}

template <int ACT, int N, int ROPE> static void go(const ExpandedArgs& x, const KvCrew& crew, const ExpandedPlan& o, hipStream_t st) {
  JoinTicket* const tickets = o.cut ? (JoinTicket*)(crew.slots + (size_t)o.slots * join_stride<EXPANDED_ROWS, N>()) : nullptr;
  k_expanded<ACT, N, ROPE><<<dim3(o.workgroups), dim3(EXPANDED_THREADS), 0, st>>>(x, crew, tickets, o.slots);
  if (o.cut) k_expanded_join<ACT, N><<<dim3(o.slots, join_split(o.slots)), dim3(JOIN_THREADS), 0, st>>>(x, crew, tickets);
}
template <int ACT> static void go(const ExpandedArgs& x, const KvCrew& crew, const ExpandedPlan& o, int n, int rope, hipStream_t st) {
  if (n == 128) rope == 64 ? go<ACT, 128, 64>(x, crew, o, st) : go<ACT, 128, 32>(x, crew, o, st);
  else rope == 64 ? go<ACT, 64, 64>(x, crew, o, st) : go<ACT, 64, 32>(x, crew, o, st);
}

static hipError_t launch_expanded(const glowq_expanded_query& p, char* ws, hipStream_t st) {
  const ExpandedPlan o = plan_expanded(p);
  ExpandedArgs x = {};
  AttendArgs& a = x.a;
  a.cache.kv_heads = p.heads;
  a.q = (const uint16_t*)p.q;
  a.out = (uint16_t*)p.out;
  a.lengths = p.lengths;
  a.starts = p.starts;
  a.ldq = p.ldq;
  a.ldo = p.ldo;
  a.n = p.n_requests;
  a.T = p.T;
  a.heads = p.heads;
  a.group = 1;
  a.max_fresh = p.max_fresh;
  a.cap = longest(p);
  a.scale = p.scale * KV_LOG2E;
  x.k = (const uint16_t*)p.k;
  x.r = (const uint16_t*)p.k_rope;
  x.v = (const uint16_t*)p.v;
  x.key_starts = p.key_starts;
  x.lhq = p.lhq;
  x.ldk = p.ldk;
  x.lhk = p.lhk;
  x.ldr = p.ldr;
  x.ldv = p.ldv;
  x.lhv = p.lhv;
  x.keys = p.keys;
  const KvCrew crew = {0, 0x7fffffff, o.shares, EXPANDED_LEAST, 0, nullptr, (float*)ws};
  p.act_dtype == GLOWQ_F16 ? go<ACT_F16>(x, crew, o, p.nope_dim, p.rope_dim, st) : go<ACT_BF16>(x, crew, o, p.nope_dim, p.rope_dim, st);
  return hipGetLastError();
}

}  // namespace glowq

using namespace glowq;
extern "C" {

glowq_status glowq_expanded_attention_workspace_bytes(const glowq_expanded_query* query, size_t* bytes) {
  if (!bytes) return GLOWQ_ERR_NULL;
  const glowq_status s = check_query(query, false);
  if (s != GLOWQ_OK) return s;
  *bytes = plan_expanded(*query).bytes;
  return GLOWQ_OK;
}

glowq_status glowq_expanded_attention(const glowq_expanded_query* query, void* workspace, size_t workspace_bytes, void* stream) {
  const glowq_status s = check_query(query, true);
  if (s != GLOWQ_OK) return s;
  if (!workspace || workspace_bytes < plan_expanded(*query).bytes) return GLOWQ_ERR_WORKSPACE;
  if ((uintptr_t)workspace & 255u) return GLOWQ_ERR_ALIGN;
  return hip_status(launch_expanded(*query, (char*)workspace, (hipStream_t)stream));
}

}  // extern "C"
