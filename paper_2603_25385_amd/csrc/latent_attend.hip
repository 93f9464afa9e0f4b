// Attention over the latent cache, absorbed: argument checks, workspace, choice of tile, launch.
#include <algorithm>
#include "attend_join.hpp"
#include "latent_attend.hpp"
#include "latent_host.hpp"

namespace glowq {

template <int ACT, int LATENT, int ROPE, int RG>
__global__ void __launch_bounds__(64 * latent_waves(RG), RG == 1 ? 1 : 2) k_latent_attend(LatentAttendArgs a, KvCrew crew, JoinTicket* tickets, int slots) {
  __shared__ LatentLds<LATENT, ROPE, RG> lds;
  KvRequest req;
  long long all, total;
  const KvPart pc = kv_cut<16 * RG, LATENT_STEP, true>(a.a, crew, blockIdx.x, req, all, total);
  if (tickets) join_leave(tickets, slots, pc, req);
  if (pc.r >= 0) latent_part<ACT, LATENT, ROPE, RG>(a, crew, pc, req, lds);
}

template <int ACT, int LATENT, int RG>
__global__ void __launch_bounds__(JOIN_THREADS) k_latent_join(LatentAttendArgs args, KvCrew crew, const JoinTicket* tickets) {
  __shared__ float scratch[JOIN_THREADS][6];
  constexpr int R = 16 * RG;
  const AttendArgs& a = args.a;
  KvRequest req;
  KvPart pc;
  if (!join_take(tickets, pc, req)) return;
  const int row0 = pc.tile * R;
  attend_join<R, LATENT>(crew, pc, min(R, req.rows - row0), R * LATENT / 4, scratch,
    [](int item, int& row, int& dim) {
      row = item / 64 % RG * 16 + (item & 15);
      dim = item / (64 * RG) * 16 + (item >> 4 & 3) * 4;
    },
    [&](float l, int row) { return kv_inverse(l, a, req, pc.r, row0 + row) * LATENT_LIFTED; },
    [&](int row, int dim, float4_t x) {
      const int i = (row0 + row) / a.group;
      uint16_t* const to = a.out + (size_t)(req.start + i) * a.ldo + (size_t)(row0 + row - i * a.group) * LATENT + dim;
      typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
      *(u32x2_t*)to = u32x2_t{kv_pack<ACT>(x[0], x[1]), kv_pack<ACT>(x[2], x[3])};
    });
}

// Steps of a part at least.  With 1, 2, 4, 8: one sequence of 900, 16 heads 12.0, 13.0, 15.2, 20.0 us; 8 of up to 500, 128 heads 20.7, 23.7, 27.5,
// 30.5; 16 of up to 2000, 128 heads 30.6, 30.7, 31.9, 40.8; a decoding step of 32 50.9, 50.8, 51.9, 60.3; longer ones and pieces the same.
// Workgroups that the machine holds at once: one on a CU, by LDS for latents of 512, by the registers of eight waves for 256 (of 16 rows, four
// waves, two would fit there: not counted on).
constexpr int LATENT_LEAST = 2;
constexpr int LATENT_PLACES = 256;
constexpr long long MOST_WORKGROUPS = 0xffffffffll / (64 * latent_waves(4));       // a launch counts its threads in 32 bits

struct LatentPlan {
  int tile;                    // blocks of 16 rows: 1, 2 or 4
  int workgroups, slots;       // at most: parts, partial results
  bool cut;                    // whether a unit can be
  size_t bytes;
};

static int longest(const glowq_latent_cache& c, const glowq_latent_query& p) {
  return (int)std::min<long long>(std::min<long long>((long long)p.table_width * c.block_tokens, p.max_length), 1 << 30);
}

static LatentPlan plan_latent(const glowq_latent_cache& c, const glowq_latent_query& p) {
  LatentPlan o = {};
  const long long rows = (long long)p.max_fresh * p.heads, all = (long long)p.T * p.heads;
  // As many rows as the largest request has, up to 64, so that keys are read once for them.  16 rows for all instead: 64 requests of 128 heads
  // 264 us for 133, eight pieces of up to 16 tokens, 128 heads 203 for 131, two long sequences of 40 heads 44.6 for 38.3, 64 of 16 heads the same; but 63 requests
  // of 16 heads beside a piece of 64 tokens 30.6 for 41.2, eight short ones of 128 heads 15.7 for 23.7.
  o.tile = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int R = 16 * o.tile;
  const long long units = std::min<long long>(p.n_requests * ((rows + R - 1) / R), all / R + std::min<long long>(p.n_requests, all));
  // Parts: kv_cut makes them larger until they fit into whole rounds, units and a quarter of a round rounded up, so that room - units is
  // 1.25 rounds at most.  A unit that is cut has two parts or more, half of them beyond its first: what leaves partial results is twice
  // room - units at most, whatever the rows.
  const long long places = LATENT_PLACES, room = places * (1 + (4 * units + places) / (4 * places));
  const long long steps = (longest(c, p) + LATENT_STEP - 1) / LATENT_STEP;
  o.cut = steps > LATENT_LEAST;
  o.workgroups = (int)std::min<long long>(o.cut ? std::min(std::max(units, room), units * steps) : units, 0x3fffffff);
  o.slots = o.cut ? (int)std::min<long long>(o.workgroups, 5 * places / 2) : 0;
  o.bytes = std::max<size_t>((size_t)o.slots * (R * (c.latent_dim + 2) * 4 + sizeof(JoinTicket)), 256);
  return o;
}

static bool bad16(const void* p) { return ((uintptr_t)p & 15u) != 0; }
static bool bad4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

static glowq_status check_query(const glowq_latent_cache* c, const glowq_latent_query* p, bool ptrs) {
  if (!c || !p) return GLOWQ_ERR_NULL;
  const glowq_status s = latent_check_cache(c, ptrs);
  if (s != GLOWQ_OK) return s;
  if (p->n_requests < 1 || p->n_requests > (1 << 20) || p->T < 1 || p->T > (1 << 20) || p->table_width < 1) return GLOWQ_ERR_SHAPE;
  if (p->heads < 1 || p->heads > 1024 || (long long)p->T * p->heads > 0x7fffffffll) return GLOWQ_ERR_SHAPE;
  if (p->max_fresh < 1 || p->max_fresh > p->T || p->max_length < 1) return GLOWQ_ERR_SHAPE;
  if (!(p->scale > 0.f) || !(p->scale <= 2e38f)) return GLOWQ_ERR_SHAPE;
  if (p->ldq < p->heads * (c->latent_dim + c->rope_dim) || p->ldo < p->heads * c->latent_dim) return GLOWQ_ERR_SHAPE;
  if (p->ldq % 8 || p->ldo % 8) return GLOWQ_ERR_UNSUPPORTED;
  if (plan_latent(*c, *p).workgroups > MOST_WORKGROUPS) return GLOWQ_ERR_SHAPE;
  if (!ptrs) return GLOWQ_OK;
  if (!p->q || !p->out || !p->table || !p->lengths || !p->starts) return GLOWQ_ERR_NULL;
  return bad16(p->q) || bad16(p->out) || bad4(p->table) || bad4(p->lengths) || bad4(p->starts) ? GLOWQ_ERR_ALIGN : GLOWQ_OK;
}

template <int ACT, int LATENT, int ROPE, int RG>
static void go(const LatentAttendArgs& a, const KvCrew& crew, const LatentPlan& o, hipStream_t st) {
  JoinTicket* const tickets = o.cut ? (JoinTicket*)(crew.slots + (size_t)o.slots * latent_stride<LATENT, RG>()) : nullptr;
  k_latent_attend<ACT, LATENT, ROPE, RG><<<dim3(o.workgroups), dim3(64 * latent_waves(RG)), 0, st>>>(a, crew, tickets, o.slots);
  if (o.cut) k_latent_join<ACT, LATENT, RG><<<dim3(o.slots, join_split(o.slots)), dim3(JOIN_THREADS), 0, st>>>(a, crew, tickets);
}
template <int ACT, int LATENT, int ROPE> static void go(const LatentAttendArgs& a, const KvCrew& crew, const LatentPlan& o, hipStream_t st) {
  if (o.tile == 1) go<ACT, LATENT, ROPE, 1>(a, crew, o, st);
  else if (o.tile == 2) go<ACT, LATENT, ROPE, 2>(a, crew, o, st);
  else go<ACT, LATENT, ROPE, 4>(a, crew, o, st);
}
template <int ACT> static void go(const LatentAttendArgs& a, const KvCrew& crew, const LatentPlan& o, int latent, int rope, hipStream_t st) {
  if (latent == 512) rope == 64 ? go<ACT, 512, 64>(a, crew, o, st) : go<ACT, 512, 32>(a, crew, o, st);
  else rope == 64 ? go<ACT, 256, 64>(a, crew, o, st) : go<ACT, 256, 32>(a, crew, o, st);
}

static hipError_t launch_latent_attention(const glowq_latent_cache& c, const glowq_latent_query& p, char* ws, hipStream_t st) {
  const LatentPlan o = plan_latent(c, p);
  LatentAttendArgs args = {};
  AttendArgs& a = args.a;
  a.cache.n_blocks = c.n_blocks;
  a.cache.kv_heads = 1;
  a.cache.block_shift = kv_shift(c.block_tokens);
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
  a.heads = a.group = p.heads;
  a.max_fresh = p.max_fresh;
  a.cap = longest(c, p);
  a.scale = p.scale * KV_LOG2E;
  args.cache = latent_view(c);
  const KvCrew crew = {0, 0x7fffffff, 1, LATENT_LEAST, 0, nullptr, (float*)ws, LATENT_PLACES};
  c.act_dtype == GLOWQ_F16 ? go<ACT_F16>(args, crew, o, c.latent_dim, c.rope_dim, st) : go<ACT_BF16>(args, crew, o, c.latent_dim, c.rope_dim, st);
  return hipGetLastError();
}

}  // namespace glowq

using namespace glowq;
extern "C" {

glowq_status glowq_latent_attention_workspace_bytes(const glowq_latent_cache* cache, const glowq_latent_query* query, size_t* bytes) {
  if (!bytes) return GLOWQ_ERR_NULL;
  const glowq_status s = check_query(cache, query, false);
  if (s != GLOWQ_OK) return s;
  *bytes = plan_latent(*cache, *query).bytes;
  return GLOWQ_OK;
}

glowq_status glowq_latent_attention(const glowq_latent_cache* cache, const glowq_latent_query* query, void* workspace, size_t workspace_bytes, void* stream) {
  const glowq_status s = check_query(cache, query, true);
  if (s != GLOWQ_OK) return s;
  if (!workspace || workspace_bytes < plan_latent(*cache, *query).bytes) return GLOWQ_ERR_WORKSPACE;
  if ((uintptr_t)workspace & 255u) return GLOWQ_ERR_ALIGN;
  return hip_status(launch_latent_attention(*cache, *query, (char*)workspace, (hipStream_t)stream));
}

}  // extern "C"
