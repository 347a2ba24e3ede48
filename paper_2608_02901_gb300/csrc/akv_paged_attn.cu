// Attention over the paged 4-bit cache: a persistent launch that reads each attended page once, and a launch that joins
// the shares of units that several CTAs worked on.
//
// Bound by HBM in principle (144 bytes a token and head at two groups a row, 2 x 16 products of 16 x 16 x 8), in practice by a
// warp's chain, which 16 warps an SM do not cover: no pipe is full (issue 55 %, ALU 47 %, tensor 34 %, DRAM 57 %).
// 4 x 131072 tokens, 8 KV heads, 4 or 8 query heads each, take 120 us (5.0 TB/s, 74 % of the measured rate), rotated 133
// (half as many products again), with 16 query rows 168, rotated 207;
// 8 x 131072 rotated tokens 235 us (5.1 TB/s).  A call has about 8 us that do not depend on the length: the plan, the
// first page numbers and copies, the joins (1021 tokens: 7 us, and 4 of the second launch).
//
// A unit is one KV head of one request (or of one query token, where each has its own pages) with up to 8 NT query
// rows.  Units are cut into tiles of 128 tokens, and the tiles of all units into equal contiguous ranges, one per CTA,
// so that one long request and many short ones fill the GPU alike (where CTAs have few tiles, see plan).  In a CTA one warp
// copies (bulk copies of whole sub-blocks into a ring of stages) and the others take the sub-blocks of 16 tokens in turn,
// without a barrier between them: each has its own running reference, sum and output, joined at the unit's end.
//
// The codes go into the tensor cores as they are.  A nibble, masked in place, is the fp16 subnormal c 2^-24 (or
// 16 c 2^-24 for the odd ones, whose partner is scaled by 1/16), so eight values cost five integer operations and no
// conversion; the products are exact in fp32, and a row's scale and minimum are applied to the sums:
//     l_i = a_i (c_i . q) + m_i sum(q),     y = sum_i (p_i a_i) c_i + sum_i p_i m_i .
// Queries are exact in fp16 (a power of two times what was given); rotated ones are fp32 and enter as a high and a
// low half.  The weights p_i a_i are rounded to fp16: relative 2^-11 for those of 2^-14 and more (a bf16 result is rounded by up
// to 2^-8).  The reference that a row's exponents p = 2^(l - reference) are taken from follows its largest p a so far, of tokens
// that it sees and of both groups: that weight is between 2^6 and 2^15, and one down to 2^-20 of it keeps its 2^-11; what
// smaller ones lose is at most 2^-31 of the largest (tokens whose scale is large but that hardly weigh, or are not seen, cost
// the others nothing).  Sums, maxima and logits are fp32.
#include <cuda_runtime.h>

#include <atomic>
#include <type_traits>

#include "akv_device.cuh"
#include "akv_paged.cuh"

namespace akv {
namespace {

constexpr int kTileTokens = 128, kTileSubs = kTileTokens / kSubTokens;
// A unit has 8 NT query rows, NT 1 or 2.  (Four were slower than two units of 16 rows that read the cache twice: 375 and
// 319 us for 32 rows a head over 4 x 131072 tokens, 53 and 40 us over 4 x 8192: 255 registers leave an SM seven warps.)
// Computing warps of a CTA, next to one that copies: an SM has room for 16 warps of 128 registers or 12 of 168 (a 17th
// and a 13th would take them down to 96 and 128, which spill).  Two CTAs per SM of 8 rows, one of 16.
AKV_HD constexpr int warps_of(int nt) { return nt == 1 ? 7 : 11; }
AKV_HD constexpr int ctas_of(int nt) { return nt == 1 ? 2 : 1; }
// Stages of the ring: what the warps are working on, and as much again on its way.
AKV_HD constexpr int stages_of(int nt) { return nt == 1 ? 4 : 6; }
// Sub-blocks that a warp takes at a time: two where the registers allow it, whose products then overlap (8 x 128K tokens:
// 284 us with one, 234 with two; with 16 rows two spill, 179 and 181 us for 4 x 131072 tokens, rotated 217 and 276).
AKV_HD constexpr int subs_of(int nt) { return nt == 1 ? 2 : 1; }
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLow = -3.402823466e38f;        // reference of a share that saw no token: below all others
constexpr float kSlack = 8.f;                   // a weight may pass its place by 2^8 before the reference moves
constexpr float kWeightLog = 7.f;               // the largest weight's place: 2^7 (at most 2^15 with the slack)
constexpr int kAlignTiles = 16;                 // tiles a CTA up to which units may get CTAs of their own
constexpr int kRowPad = kD + 4;                 // floats between rows of the joined outputs

struct AttnArgs {
  PagedView v;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t qb, qt, qh, ob, ot, oh;
  const int32_t* sel;
  const int32_t* count;
  int4* desc;     // [grid]: unit that starts in a CTA and goes on: group, index in it, last CTA
  float* slots;   // [grid][2] partial results of 8 NT rows
  float scale;    // sm_scale log2(e)
  int T, top;
  int rows;       // query rows of a unit in all (T G, or G)
  int n_blocks;   // units that share them
  int groups;     // requests, or (request, query token, head) with a selection
  int per_group;  // units of a group
};

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The larger of three (a NaN is left out).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float word_scale(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)w)); }
__device__ __forceinline__ float word_min(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
__device__ __forceinline__ uint32_t comp(const uint4& x, int j) { return j == 0 ? x.x : j == 1 ? x.y : j == 2 ? x.z : x.w; }
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }  // -126 .. 127

// Tokens that a group's units go through, in the order of its tiles.
struct Group {
  int b, t, h;   // (t, h: with a selection)
  int tokens;    // positions its tiles cover: the request's, or the kept pages'
  int sees;      // tokens that may be attended at all
};
template <bool SEL>
__device__ __forceinline__ Group group_of(const AttnArgs& a, int gi) {
  Group g;
  if (SEL) {
    g.h = gi % a.v.H;
    g.t = gi / a.v.H % a.T;
    g.b = gi / a.v.H / a.T;
    g.sees = max(0, held_tokens(a.v, g.b) - a.T + 1 + g.t);
    g.tokens = min(max(a.count[gi], 0), a.top) << a.v.page_log;
  } else {
    g.b = gi;
    g.t = g.h = 0;
    g.sees = g.tokens = held_tokens(a.v, gi);
  }
  return g;
}
__device__ __forceinline__ int tiles_of(const Group& g) { return max(1, (g.tokens + kTileTokens - 1) / kTileTokens); }

// Where a CTA's range of tiles begins and how long it is.
struct Range {
  int64_t lo, hi, total;
  int ctas, shares;  // shares: into how many CTAs' parts the CTA's one unit is cut; 0: the CTA goes over tiles of several
};
// The place of a tile: unit `index` of group `gi`, tile `ti` of the unit.
template <bool SEL>
struct Cursor {
  int gi, index, ti, tiles;
  Group g;
  __device__ __forceinline__ void open(const AttnArgs& a) {
    g = group_of<SEL>(a, gi);
    tiles = tiles_of(g);
  }
  // the first tile of the next unit
  __device__ __forceinline__ void next_unit(const AttnArgs& a) {
    ti = 0;
    if (++index == a.per_group) {
      index = 0;
      ++gi;
      if (gi < a.groups) open(a);
    }
  }
};

struct PlanSmem {
  int64_t part[2][16];  // sums of the warps
  int most[16];
  int place[10];        // the CTA's place: what the thread that finds it writes down
};
// Sum over the CTA's threads before this one; *total: over all.  All threads call it.
template <int kThreads>
__device__ __forceinline__ int64_t sum_before(int64_t x, int64_t* part, int64_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t inc = x;
#pragma unroll
  for (int h = 1; h < 32; h *= 2) {
    const int64_t o = __shfl_up_sync(0xffffffffu, inc, h);
    if (lane >= h) inc += o;
  }
  if (lane == 31) part[warp] = inc;
  __syncthreads();
  int64_t before = inc - x, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += part[w];
    all += part[w];
  }
  *total = all;
  return before;
}

// Every thread: this CTA's range and its first tile.
template <int kThreads, bool SEL>
__device__ __forceinline__ Range plan(const AttnArgs& a, PlanSmem& S, Cursor<SEL>& c) {
  const int tid = threadIdx.x, strip = (a.groups + kThreads - 1) / kThreads;  // groups of a thread
  const int g0 = tid * strip, g1 = min(a.groups, g0 + strip);
  Cursor<SEL> mine;  // the thread's first group
  mine.gi = g0;
  int64_t tiles = 0;
  if (g0 < g1) {
    mine.open(a);
    tiles = mine.tiles;
    for (int gi = g0 + 1; gi < g1; ++gi) tiles += tiles_of(group_of<SEL>(a, gi));
  }
  Range r;
  r.shares = 0;
  r.lo = r.hi = 0;
  tiles *= a.per_group;
  int64_t here = tiles, before = sum_before<kThreads>(tiles, S.part[0], &r.total);
  r.ctas = (int)min((int64_t)gridDim.x, r.total);
  // Where a CTA has few tiles, the second unit of one that gets parts of two costs as much as some tiles: then every unit
  // has CTAs of its own, if the longest share stays as short but for a tile (32 x 1000 tokens of 8 heads: 19.9 -> 15.4 us a
  // call, 32 x 200: 11.8 -> 8.9, 8 x 1021: 11.7 -> 10.1; a call that it does not change takes 0.2 us more).
  const int even = (int)min((int64_t)(1 << 20), (r.total + gridDim.x - 1) / gridDim.x);
  auto shares_of = [&](int t) { return min(t, max(1, (int)(gridDim.x * (uint32_t)t / (uint32_t)r.total))); };
  if (even <= kAlignTiles && strip == 1) {
    const int s = tiles ? shares_of(mine.tiles) : 0;
    int most = __reduce_max_sync(0xffffffffu, s ? (mine.tiles + s - 1) / s : 0);
    if ((tid & 31) == 0) S.most[tid >> 5] = most;
    int64_t all;
    const int64_t cut = (int64_t)s * a.per_group, cut_before = sum_before<kThreads>(cut, S.part[1], &all);
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) most = max(most, S.most[w]);
    if (all <= gridDim.x && most <= even + 1) {
      r.shares = 1;
      r.ctas = (int)all;
      here = cut;
      before = cut_before;
    }
  }
  if ((int)blockIdx.x >= r.ctas) return r;
  const int64_t want = r.shares ? blockIdx.x : blockIdx.x * r.total / r.ctas;  // the CTA's share, or its first tile
  if (want >= before && want < before + here) {  // one thread's groups hold it
    int64_t rest = want - before;
    while (!r.shares && rest >= (int64_t)mine.tiles * a.per_group) {
      rest -= (int64_t)mine.tiles * a.per_group;
      ++mine.gi;
      mine.open(a);
    }
    int each = r.shares ? shares_of(mine.tiles) : mine.tiles, i = (int)(rest % each);
    S.place[0] = mine.gi, S.place[1] = (int)(rest / each), S.place[2] = i, S.place[3] = mine.tiles, S.place[4] = mine.g.b;
    S.place[5] = mine.g.t, S.place[6] = mine.g.h, S.place[7] = mine.g.tokens, S.place[8] = mine.g.sees, S.place[9] = each;
  }
  __syncthreads();
  c.gi = S.place[0], c.index = S.place[1], c.ti = S.place[2], c.tiles = S.place[3], c.g.b = S.place[4];
  c.g.t = S.place[5], c.g.h = S.place[6], c.g.tokens = S.place[7], c.g.sees = S.place[8];
  if (r.shares) {
    const int i = c.ti;
    r.shares = S.place[9];
    r.lo = c.ti = i * c.tiles / r.shares;
    r.hi = (i + 1) * c.tiles / r.shares;
  } else {
    r.lo = want;
    r.hi = (blockIdx.x + 1) * r.total / r.ctas;
  }
  return r;
}

template <int NT>
struct Smem {
  static constexpr int kWarps = warps_of(NT), kThreads = 32 * (kWarps + 1), kStages = stages_of(NT);
  alignas(128) uint8_t stage[kStages][kTileSubs * 2304];
  alignas(16) uint4 frag[2][NT][4][32];     // query operand: high, low halves
  float red[kWarps][8 * NT][kRowPad];       // the warps' outputs at a unit's end
  float red_m[kWarps][8 * NT], red_l[kWarps][8 * NT];
  float qsum[8 * NT][2];                    // sums of a query row over each group of dimensions
  float qscale[8 * NT];                     // what its products count
  int pos[kStages][kTileSubs];              // first token of each sub-block; -1: none, -2: a page outside the pool
  uint32_t tile[kStages];                   // the CTA's tile that the stage holds or waits for
  int cursor[kWarps][10];                   // a warp's place, kept here while it works on a unit (registers are short)
  PlanSmem plan;
  int64_t range_lo, range_total;
  int range_shares;
  uint64_t full[kStages], empty[kStages];
  int failed;
};

constexpr int kConsumerBar = 1;

template <int NG, int NT, bool HILO, bool SEL>
__global__ void __launch_bounds__(32 * (warps_of(NT) + 1), ctas_of(NT)) akv_paged_attn_kernel(const __grid_constant__ AttnArgs a) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  Smem<NT>& S = *reinterpret_cast<Smem<NT>*>(smem_raw);
  constexpr uint32_t kSub = 2048 + 128 * NG;
  constexpr int kRows = 8 * NT, kWarps = warps_of(NT), kThreads = 32 * (kWarps + 1), NS = subs_of(NT), kStages = stages_of(NT);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const PagedView& v = a.v;

  launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&S.full[s]), 1);
      mbar_init(smem_u32(&S.empty[s]), kTileSubs / NS);
      S.tile[s] = ~0u;
    }
    S.failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  wait_for_stream();
  Cursor<SEL> c;
  const Range r = plan<kThreads, SEL>(a, S.plan, c);  // (its barriers order the initialisation too)
  if (tid == 0) a.desc[blockIdx.x] = make_int4(-1, 0, 0, 0);
  if (r.lo >= r.hi) return;
  volatile int* failed = &S.failed;

  if (warp == kWarps) {
    // ---- the copying warp: lane k < 8 sees to sub-block k of a tile, the first lane of a page copies its sub-blocks
    const int per_page = min(kTileSubs, 1 << (v.page_log - 4));
    // the bulk copies read what launches before this one wrote with ordinary stores
    asm volatile("fence.proxy.async.global;" ::: "memory");
    int stage = 0;
    uint32_t phase = 1;  // the first pass over the ring waits for nobody
    // What the next tiles need is under way while a tile waits for its stage, and nothing looks at it before its turn:
    // the table's page numbers kAhead tiles before, with a selection its entries as much earlier.
    constexpr int kAhead = 3;
    struct Place {
      int j, off, b, h, sees;  // the lane's sub-block: table position (-1: none), first token in its page; request, head
    };
    struct Look {
      int at, page, h;  // first token, -1: none; its page as the table says; head
    };
    int64_t looked = r.lo;
    auto next_place = [&]() {
      Place p{-1, 0, 0, 0, 0};
      if (looked >= r.hi) return p;
      if (looked++ > r.lo && ++c.ti == c.tiles) c.next_unit(a);
      const int i = c.ti * kTileTokens + lane * kSubTokens;
      p.b = c.g.b, p.h = SEL ? c.g.h : c.index / a.n_blocks, p.sees = c.g.sees;
      if (lane >= kTileSubs || i >= c.g.tokens) return p;
      p.off = i & ((1 << v.page_log) - 1);
      p.j = SEL ? a.sel[(int64_t)c.gi * a.top + (i >> v.page_log)] : i >> v.page_log;
      return p;
    };
    auto look = [&](const Place& p) {
      Look l{-1, -1, p.h};
      if ((uint32_t)p.j >= (uint32_t)v.max_pages) return l;
      const int at = (p.j << v.page_log) + p.off;
      if (at >= p.sees) return l;
      l.at = at;
      l.page = v.table[(int64_t)p.b * v.table_stride + p.j];
      return l;
    };
    Place places[kAhead];
    Look looks[kAhead];
    if (SEL) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) places[i] = next_place();
    }
    auto look_next = [&]() {
      if (!SEL) return look(next_place());
      const Look l = look(places[0]);
#pragma unroll
      for (int i = 0; i + 1 < kAhead; ++i) places[i] = places[i + 1];
      places[kAhead - 1] = next_place();
      return l;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) looks[i] = look_next();
    int64_t end = r.hi;
    for (int64_t k = r.lo; k < end; ++k) {
      const Look now = looks[0];
#pragma unroll
      for (int i = 0; i + 1 < kAhead; ++i) looks[i] = looks[i + 1];
      looks[kAhead - 1] = look_next();
      const int page0 = now.page, h0 = now.h;
      const int pos0 = now.at < 0 ? -1 : (uint32_t)page0 < (uint32_t)v.n_pages ? now.at : -2;
      if (!mbar_wait_w(smem_u32(&S.empty[stage]), phase)) {
        if (lane == 0) *failed = 1;
        end = k;
        break;
      }
      const uint32_t there = __ballot_sync(0xffffffffu, pos0 >= 0);
      if (lane < kTileSubs) S.pos[stage][lane] = pos0;
      if (lane == kTileSubs) *(volatile uint32_t*)&S.tile[stage] = (uint32_t)(k - r.lo);
      __syncwarp();
      const uint32_t bar = smem_u32(&S.full[stage]);
      if (lane == 0) mbar_expect_tx(bar, (uint32_t)__popc(there) * kSub);
      __syncwarp();
      if (pos0 >= 0 && lane % per_page == 0) {
        const uint32_t n = (uint32_t)__popc(there >> lane & ((1u << per_page) - 1));
        bulk_g2s(smem_u32(&S.stage[stage][lane * kSub]), block_of(v, page0, h0) + (uint64_t)((pos0 & ((1 << v.page_log) - 1)) >> 4) * kSub,
                 n * kSub, bar);
      }
      if (++stage == kStages) stage = 0, phase ^= 1;
    }
    // shared memory is the copies' until the last have landed, also where a warp has given up
    for (uint32_t n = (uint32_t)(end - r.lo), k = n > kStages ? n - kStages : 0; k < n; ++k)
      if (!mbar_wait_w(smem_u32(&S.full[k % kStages]), k / kStages & 1)) break;
    return;
  }

  // ---- the computing warps
  const int g8 = lane >> 2, t4 = lane & 3;
  const uint32_t range = (uint32_t)(r.hi - r.lo);  // tiles of the CTA
  auto keep = [&](const Cursor<SEL>& x) {
    __syncwarp();
    if (lane == 0) {
      volatile int* to = S.cursor[warp];
      to[0] = x.gi, to[1] = x.index, to[2] = x.ti, to[3] = x.tiles, to[4] = x.g.b, to[5] = x.g.t, to[6] = x.g.h;
      to[7] = x.g.tokens, to[8] = x.g.sees;
    }
    __syncwarp();
  };
  auto kept = [&]() {
    const volatile int* from = S.cursor[warp];
    Cursor<SEL> x;
    x.gi = from[0], x.index = from[1], x.ti = from[2], x.tiles = from[3], x.g.b = from[4], x.g.t = from[5], x.g.h = from[6];
    x.g.tokens = from[7], x.g.sees = from[8];
    return x;
  };
  auto tiles_here = [&](const Cursor<SEL>& x, uint32_t at) { return (int)min((uint32_t)(x.tiles - x.ti), range - at); };
  keep(c);
  if (tid == 0) S.range_lo = r.lo, S.range_total = r.total, S.range_shares = r.shares;  // (read by the same thread)
  uint32_t at = 0;  // tiles done
  while (at < range) {
    int row0, n_tiles, sees, all_see;
    {
    const Cursor<SEL> cu = kept();
    const int b = cu.g.b, h = SEL ? cu.g.h : cu.index / a.n_blocks;
    row0 = (SEL ? cu.index : cu.index % a.n_blocks) * kRows;
    const int n_rows = min(kRows, a.rows - row0);
    n_tiles = tiles_here(cu, at);
    sees = cu.g.sees;
    all_see = SEL ? sees : sees - a.T + 1;  // every row of the unit sees the tokens before this one

    // queries: a warp per row, four dimensions a lane
    constexpr int kTurns = (kRows + kWarps - 1) / kWarps;
    float qx[kTurns][4], big[kTurns];
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int rr = warp + kWarps * i;
#pragma unroll
      for (int e = 0; e < 4; ++e) qx[i][e] = 0.f;
      big[i] = 0.f;
      if (rr < n_rows) {
        const int t = SEL ? cu.g.t : (row0 + rr) / v.G, g = SEL ? row0 + rr : (row0 + rr) % v.G;
        const uint16_t* row = a.q + b * a.qb + t * a.qt + (int64_t)(h * v.G + g) * a.qh + 4 * lane;
        if (((uintptr_t)row & 7) == 0) {
          const uint2 w = *(const uint2*)row;
          qx[i][0] = row_to_float((uint16_t)w.x, v.half);
          qx[i][1] = row_to_float((uint16_t)(w.x >> 16), v.half);
          qx[i][2] = row_to_float((uint16_t)w.y, v.half);
          qx[i][3] = row_to_float((uint16_t)(w.y >> 16), v.half);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) qx[i][e] = row_to_float(row[e], v.half);
        }
      }
      if (HILO) {  // q' = H (s o q) / 16
#pragma unroll
        for (int e = 0; e < 4; ++e) qx[i][e] = __uint_as_float(__float_as_uint(qx[i][e]) ^ sign_flip(v, 4 * lane + e));
        wht_32x4(qx[i], lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) qx[i][e] *= 0.0625f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = fabsf(qx[i][e]);
        if (x <= 3.402823466e38f) big[i] = fmaxf(big[i], x);  // an infinite or NaN row spoils itself alone
      }
      big[i] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(big[i])));
    }
    named_sync(kConsumerBar, 32 * kWarps);  // (also: every warp is through with the unit before)
    // A row times 2^(14 - e), e its own exponent: below 2^14, and exact in fp16 down to 2^-23 of that.  (With one e for the
    // rows of a unit, 233.5 us for 235.5 over 8 x 128K tokens, a large row, padding say, took the others' values below fp16's range.)
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int rr = warp + kWarps * i;
      if (rr >= kRows) break;
      const int e = min(max((int)(__float_as_uint(big[i]) >> 23) - 126, -100), 128);
      const float up = pow2(14 - e);
      if (lane == 0) S.qscale[rr] = a.scale * pow2(e - 10) * 1048576.f;  // codes count 2^-24, queries 2^(14 - e)
      float sum = (qx[i][0] + qx[i][1]) + (qx[i][2] + qx[i][3]);
#pragma unroll
      for (int m = 1; m < 32 / NG; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
      if (lane % (32 / NG) == 0) S.qsum[rr][lane / (32 / NG)] = sum * a.scale;
      uint4 f[HILO ? 2 : 1];
#pragma unroll
      for (int lo = 0; lo < (HILO ? 2 : 1); ++lo) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // nibble e: odd ones stand for 16 times their value
          const float x = qx[i][e] * (e & 1 ? up * 0.0625f : up);
          const float hi = __half2float(__float2half_rn(x));
          const float mine = lo ? x - hi : x;
          const float other = __shfl_xor_sync(0xffffffffu, mine, 1);
          w[e] = lane & 1 ? half2_bits(other, mine) : half2_bits(mine, other);
        }
        f[lo] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      // lanes 2 x and 2 x + 1 hold dimensions 8 x ..: word j = x / 4, operand lane 4 row + x % 4
      const int to = 4 * (rr & 7) + (lane >> 1 & 3);
      if (!(lane & 1)) S.frag[0][rr >> 3][lane >> 3][to] = f[0];
      if (HILO && (lane & 1)) S.frag[1][rr >> 3][lane >> 3][to] = f[HILO ? 1 : 0];
    }
    named_sync(kConsumerBar, 32 * kWarps);
    }
    // What goes with a lane's rows, 2 t4 and 2 t4 + 1 of each eight: with 16 rows it stays in shared memory, registers are short
    // (4 x 128K tokens, 4 query tokens each: 168 us for 183).
    float own_sum[2][NG], own_scale[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      own_scale[x] = S.qscale[2 * t4 + x];
#pragma unroll
      for (int g = 0; g < NG; ++g) own_sum[x][g] = S.qsum[2 * t4 + x][g];
    }
    auto row_sum = [&](int nt, int x, int g) { return NT == 1 ? own_sum[x][g] : S.qsum[8 * nt + 2 * t4 + x][g]; };
    auto row_scale = [&](int nt, int x) { return NT == 1 ? own_scale[x] : S.qscale[8 * nt + 2 * t4 + x]; };

    float acc[NT][8][4], sum[NT][2], mins[NT][2][NG], ref[NT][2];
    int e_s = 103;  // the values' scales so far are at most 2^(e_s - 127)
    float most = kNegInf;  // up to here l - reference has room with any scale so far, 15 - (e_s - 127); no reference yet
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int mt = 0; mt < 8; ++mt)
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[nt][mt][x] = 0.f;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        sum[nt][x] = 0.f;
        ref[nt][x] = 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g) mins[nt][x][g] = 0.f;
      }
    }
    auto spoil = [&]() {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sum[nt][0] = sum[nt][1] = __int_as_float(0x7fffffff);
    };

    for (int item = warp; item < n_tiles * (kTileSubs / NS); item += kWarps) {
      const int sub = item % (kTileSubs / NS) * NS;
      const uint32_t tile = at + item / (kTileSubs / NS);  // of the CTA's
      const int stage = tile % kStages;
      const uint32_t bar = smem_u32(&S.full[stage]), parity = tile / kStages & 1;
      // A warp passes over tiles that it has no part of, so the parity alone could be that of a phase long ago: the stage
      // is this tile's once its number is (read first), and then the phase is the right one.
      auto ready = [&]() {
        const bool mine = *(volatile uint32_t*)&S.tile[stage] == tile;
        return __all_sync(0xffffffffu, mbar_try(bar, parity) && mine);
      };
      if (!ready()) {
        bool there = false;
        const unsigned long long t0 = global_ns();
        for (unsigned i = 1; !there && !warp_failed(failed); ++i) {
          there = ready();
          if ((i & 63u) == 0 && __shfl_sync(0xffffffffu, global_ns() - t0 >= kWaitNs ? 1 : 0, 0)) break;
        }
        if (!there) {
          *failed = 1;
          spoil();
          break;
        }
      }
      int pos[NS];
      bool none = true, edge = false, outside = false;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        pos[i] = S.pos[stage][sub + i];
        outside = outside || pos[i] == -2;
        none = none && pos[i] < 0;
        if (pos[i] < 0) pos[i] = 1 << 30;  // (nobody sees its tokens)
        edge = edge || pos[i] + kSubTokens > all_see;
      }
      if (outside) spoil();
      if (none) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.empty[stage]));
        continue;
      }
      const uint32_t sb = smem_u32(&S.stage[stage][sub * kSub]);

      // logits of tokens g8 and g8 + 8, query rows 2 t4 and 2 t4 + 1 (log2 units), less the rows' references
      auto words_at = [&](int i, int x, int side, uint32_t (&w)[NG]) {  // a token's scales and minima
        const uint8_t* at = &S.stage[stage][(sub + i) * kSub + 2048 + 8 * NG * (g8 + 8 * x) + 4 * NG * side];
        if (NG == 2) {
          const uint2 y = *(const uint2*)at;
          w[0] = y.x, w[NG - 1] = y.y;
        } else {
          w[0] = *(const uint32_t*)at;
        }
      };
      float l[NS][NT][4];
      {
        uint4 kc[NS][2];
        uint32_t kw[NS][2][NG];
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          kc[i][0] = lds128(sb + i * kSub + 16 * lane);
          kc[i][1] = lds128(sb + i * kSub + 512 + 16 * lane);
#pragma unroll
          for (int x = 0; x < 2; ++x) words_at(i, x, 0, kw[i][x]);
        }
        // (sums of 64 dimensions each, the low halves first: the tensor cores cut what they add off at the sum's size)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float s[NS][NT][4];
#pragma unroll
          for (int lo = HILO ? 1 : 0; lo >= 0; --lo)
#pragma unroll
            for (int j = 2 * half; j < 2 * half + 2; ++j)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                const uint4 q = S.frag[lo][nt][j][lane];
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                  const uint32_t x0 = comp(kc[i][0], j), x1 = comp(kc[i][1], j), y0 = x0 >> 8, y1 = x1 >> 8;
                  float(&d)[4] = s[i][nt];
                  if (lo == (HILO ? 1 : 0) && j == 2 * half)
                    mma_16816_first(d, x0 & 0x000f000fu, x1 & 0x000f000fu, y0 & 0x000f000fu, y1 & 0x000f000fu, q.x, q.z);
                  else
                    mma_16816(d, x0 & 0x000f000fu, x1 & 0x000f000fu, y0 & 0x000f000fu, y1 & 0x000f000fu, q.x, q.z);
                  mma_16816(d, x0 & 0x00f000f0u, x1 & 0x00f000f0u, y0 & 0x00f000f0u, y1 & 0x00f000f0u, q.y, q.w);
                }
              }
#pragma unroll
          for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const float unit = word_scale(kw[i][x >> 1][half * (NG - 1)]);
                l[i][nt][x] = half ? fmaf(unit, s[i][nt][x], l[i][nt][x]) : unit * s[i][nt][x];
              }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              float y = fmaf(word_min(kw[i][x >> 1][0]), row_sum(nt, x & 1, 0), -ref[nt][x & 1]);
              if (NG == 2) y = fmaf(word_min(kw[i][x >> 1][NG - 1]), row_sum(nt, x & 1, NG - 1), y);
              l[i][nt][x] = fmaf(l[i][nt][x], row_scale(nt, x & 1), y);
            }
      }
      float vs[NS][2][NG], vm[NS][2][NG];
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint32_t w[NG];
          words_at(i, x, 1, w);
#pragma unroll
          for (int g = 0; g < NG; ++g) vs[i][x][g] = word_scale(w[g]), vm[i][x][g] = word_min(w[g]);
        }
      uint4 vc[NS][2];
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        vc[i][0] = lds128(sb + i * kSub + 1024 + 16 * lane);
        vc[i][1] = lds128(sb + i * kSub + 1536 + 16 * lane);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&S.empty[stage]));  // what is needed is in registers
      if (edge) {  // tokens past the request, and those that a draft's earlier rows do not see
#pragma unroll
        for (int i = 0; i < NS; ++i) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const bool held = pos[i] + g8 + 8 * x < sees;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              vs[i][x][g] = held ? vs[i][x][g] : 0.f;
              vm[i][x][g] = held ? vm[i][x][g] : 0.f;
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int row = row0 + 8 * nt + 2 * t4 + (x & 1);
              if (pos[i] + g8 + 8 * (x >> 1) >= (SEL ? sees : min(sees, all_see + row / v.G))) l[i][nt][x] = kNegInf;
            }
        }
      }

      // references move only where a weight would pass its room
      float top_s = 0.f, top_l = kNegInf;  // (a NaN is left out)
#pragma unroll
      for (int i = 0; i < NS; ++i) {
#pragma unroll
        for (int g = 0; g < NG; ++g) top_s = max3(top_s, vs[i][0][g], vs[i][1][g]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) top_l = max3(max3(l[i][nt][0], l[i][nt][1], l[i][nt][2]), l[i][nt][3], top_l);
      }
      if (__any_sync(0xffffffffu, top_l > most || top_s > __int_as_float(e_s << 23))) {
        e_s = min(max(e_s, (int)(__reduce_max_sync(0xffffffffu, __float_as_uint(top_s)) >> 23) + 1), 254);
        // (a row that sees none of its warp's first tokens sees none of the later ones: it keeps its reference)
        const bool first = most == kNegInf;
        most = kSlack + kWeightLog - (float)(e_s - 127);
        float above[NS][2];  // log2 of a power of two above the token's scales, of 2^-24 (the smallest) for scales of 0
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float a = NG == 2 ? fmaxf(vs[i][x][0], vs[i][x][NG - 1]) : vs[i][x][0];
            above[i][x] = (float)(min(max((int)(__float_as_uint(a) >> 23), 102), 142) - 126);
          }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float m = kNegInf;
#pragma unroll
            for (int i = 0; i < NS; ++i) m = max3(m, l[i][nt][x] + above[i][0], l[i][nt][x + 2] + above[i][1]);
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
            // the row's largest weight goes to its place where it has passed its room
            const float up = m > (first ? kNegInf : kSlack + kWeightLog) ? m - kWeightLog : 0.f;
            ref[nt][x] += up;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
              l[i][nt][x] -= up;
              l[i][nt][x + 2] -= up;
            }
            const float f = first ? 0.f : exp2_fast(-up);
            sum[nt][x] *= f;
#pragma unroll
            for (int g = 0; g < NG; ++g) mins[nt][x][g] *= f;
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) {
              acc[nt][mt][x] *= f;
              acc[nt][mt][x + 2] *= f;
            }
          }
      }

#pragma unroll
      for (int i = 0; i < NS; ++i) {
        uint32_t w0[NT][NG], w1[NT][NG];
        auto weigh = [&](auto edge_) {
          constexpr bool kEdge = decltype(edge_)::value;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float p[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              p[x] = exp2_fast(l[i][nt][x]);
              sum[nt][x & 1] += p[x];
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              float u[4];
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                u[x] = p[x] * vs[i][x >> 1][g];
                float m = vm[i][x >> 1][g];
                if (kEdge && l[i][nt][x] == kNegInf) u[x] = m = 0.f;  // a NaN that this row does not see
                mins[nt][x & 1][g] = fmaf(p[x], m, mins[nt][x & 1][g]);
              }
              const uint32_t h0 = half2_bits(u[0], u[1]), h1 = half2_bits(u[2], u[3]);
              if (v.half) {
                // An fp16 result is as fine as the weights: what their rounding takes from a code of 7.5, the middle, goes to
                // the sums of the minima, so that only a code's distance from the middle feels it.
                mins[nt][0][g] = fmaf(7.5f, (u[0] - word_scale(h0)) + (u[2] - word_scale(h1)), mins[nt][0][g]);
                mins[nt][1][g] = fmaf(7.5f, (u[1] - word_min(h0)) + (u[3] - word_min(h1)), mins[nt][1][g]);
              }
              w0[nt][g] = transpose_8x8(h0);
              w1[nt][g] = transpose_8x8(h1);
            }
          }
        };
        if (edge) weigh(std::true_type{});
        else weigh(std::false_type{});
        // outputs: rows of the product are dimensions 64 s + 8 g8 + 4 u + n of word 2 s + u
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t x0 = comp(vc[i][0], j), x1 = comp(vc[i][1], j), y0 = x0 >> 8, y1 = x1 >> 8;
          constexpr int kShift = NG == 2 ? 1 : 2;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma_16816(acc[nt][2 * j], x0 & 0x000f000fu, y0 & 0x000f000fu, x1 & 0x000f000fu, y1 & 0x000f000fu, w0[nt][j >> kShift],
                      w1[nt][j >> kShift]);
            mma_16816(acc[nt][2 * j + 1], x0 & 0x00f000f0u, y0 & 0x00f000f0u, x1 & 0x00f000f0u, y1 & 0x00f000f0u, w0[nt][j >> kShift],
                      w1[nt][j >> kShift]);
          }
        }
      }
    }

    // ---- the unit's end, or the range's: the warps' outputs are joined
    {
      const float down = 16777216.f, down16 = 1048576.f;  // codes count 2^-24, odd ones 2^-20
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float s = sum[nt][x], m[NG];
#pragma unroll
          for (int sh = 4; sh < 32; sh *= 2) s += __shfl_xor_sync(0xffffffffu, s, sh);
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            m[g] = mins[nt][x][g];
#pragma unroll
            for (int sh = 4; sh < 32; sh *= 2) m[g] += __shfl_xor_sync(0xffffffffu, m[g], sh);
          }
          const int row = 8 * nt + 2 * t4 + x;
          if (g8 == 0) S.red_m[warp][row] = s == 0.f ? kLow : ref[nt][x], S.red_l[warp][row] = s;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float add = m[NG == 2 ? j >> 1 : 0];
            const float4 y = make_float4(fmaf(acc[nt][2 * j][x], down, add), fmaf(acc[nt][2 * j + 1][x], down16, add),
                                         fmaf(acc[nt][2 * j][x + 2], down, add), fmaf(acc[nt][2 * j + 1][x + 2], down16, add));
            *(float4*)&S.red[warp][row][64 * (j >> 1) + 8 * g8 + 4 * (j & 1)] = y;
          }
        }
    }
    named_sync(kConsumerBar, 32 * kWarps);
    Cursor<SEL> cu = kept();
    const int b = cu.g.b, h = SEL ? cu.g.h : cu.index / a.n_blocks, n_rows = min(kRows, a.rows - row0);
    const bool from_start = cu.ti == 0, to_end = cu.ti + n_tiles == cu.tiles, whole = from_start && to_end;
    float* slot = a.slots + (2 * (size_t)blockIdx.x + (from_start ? 1 : 0)) * paged_slot_floats(kRows);
#pragma unroll 1
    for (int rr = warp; rr < n_rows; rr += kWarps) {
      float m = kLow, l = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) m = fmaxf(m, S.red_m[w][rr]);
      float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_fast(S.red_m[w][rr] - m);
        const float4 x = *(const float4*)&S.red[w][rr][4 * lane];
        l = fmaf(f, S.red_l[w][rr], l);
        y[0] = fmaf(f, x.x, y[0]);
        y[1] = fmaf(f, x.y, y[1]);
        y[2] = fmaf(f, x.z, y[2]);
        y[3] = fmaf(f, x.w, y[3]);
      }
      if (!whole) {
        *(float4*)(slot + rr * kD + 4 * lane) = make_float4(y[0], y[1], y[2], y[3]);
        if (lane == 0) slot[kRows * kD + 2 * rr] = m, slot[kRows * kD + 2 * rr + 1] = l;
        continue;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] *= inv;
      if (HILO) {
        wht_32x4(y, lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = __uint_as_float(__float_as_uint(y[e] * 0.0625f) ^ sign_flip(v, 4 * lane + e));
      }
      const int t = SEL ? cu.g.t : (row0 + rr) / v.G, g = SEL ? row0 + rr : (row0 + rr) % v.G;
      uint16_t* row = a.out + b * a.ob + t * a.ot + (int64_t)(h * v.G + g) * a.oh + 4 * lane;
#pragma unroll
      for (int e = 0; e < 4; ++e) row[e] = float_to_row(y[e], v.half);
      if (a.lse && lane == 0)
        a.lse[((int64_t)b * a.T + t) * (v.H * v.G) + h * v.G + g] = l == 0.f ? kNegInf : (m + log2f(l)) * 0.693147180559945f;
    }
    if (from_start && !to_end && tid == 0) {
      // the CTA of the unit's last tile: (x + 1) ctas - 1 over the tiles of all
      const int64_t total = S.range_total, last = S.range_lo + at + cu.tiles - 1;
      const int64_t ctas = min((int64_t)gridDim.x, total);
      const int at_last = S.range_shares ? blockIdx.x + S.range_shares - 1 : (int)(((last + 1) * ctas - 1) / total);
      a.desc[blockIdx.x] = make_int4(cu.gi, cu.index, at_last, 1);
    }
    at += (uint32_t)n_tiles;
    if (at < range) {
      cu.next_unit(a);
      keep(cu);
    }
  }
}

// Joins the shares of the unit that starts in CTA blockIdx.x and goes on in others: one CTA per query row, its warps
// take the shares in turn.  Latency alone: 4 to 6 us after the attention's last CTA by itself, about 3 as its dependent.
// (Joined by the CTA that ends last instead, 8 shares of 8 rows took 11 us a call where this takes 8, 64 shares 27 for 10.)
constexpr int kJoinWarps = 8;
template <bool SEL>
__global__ void __launch_bounds__(32 * kJoinWarps) akv_paged_join_kernel(const __grid_constant__ AttnArgs a, int kRows) {
  launch_dependents();
  wait_for_stream();
  const int4 d = a.desc[blockIdx.x];
  if (d.w <= 0) return;
  const PagedView& v = a.v;
  const int rr = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = (SEL ? d.y : d.y % a.n_blocks) * kRows + rr;
  if (row >= a.rows) return;
  const int first = blockIdx.x, n = d.z - first + 1;
  const size_t floats = paged_slot_floats(kRows);
  auto slot = [&](int i) { return a.slots + (i == 0 ? 2 * (size_t)first + 1 : 2 * (size_t)(first + i)) * floats; };
  __shared__ float sm[kJoinWarps], sl[kJoinWarps], sy[kJoinWarps][kD];
  float m = kLow, l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = warp; i0 < n; i0 += 4 * kJoinWarps) {
    float4 x[4];
    float mm[4], ll[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * kJoinWarps;
      mm[u] = kLow, ll[u] = 0.f, x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < n) {
        const float* s = slot(i);
        x[u] = *(const float4*)(s + rr * kD + 4 * lane);
        const float2 ml = *(const float2*)(s + kRows * kD + 2 * rr);
        mm[u] = ml.x, ll[u] = ml.y;
      }
    }
    const float mn = fmaxf(m, fmaxf(fmaxf(mm[0], mm[1]), fmaxf(mm[2], mm[3])));
    const float f = exp2_fast(m - mn);
    m = mn;
    l *= f;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float w = exp2_fast(mm[u] - m);
      l = fmaf(w, ll[u], l);
      y[0] = fmaf(w, x[u].x, y[0]);
      y[1] = fmaf(w, x[u].y, y[1]);
      y[2] = fmaf(w, x[u].z, y[2]);
      y[3] = fmaf(w, x[u].w, y[3]);
    }
  }
  *(float4*)&sy[warp][4 * lane] = make_float4(y[0], y[1], y[2], y[3]);
  if (lane == 0) sm[warp] = m, sl[warp] = l;
  __syncthreads();
  if (warp) return;
  for (int w = 1; w < kJoinWarps; ++w) m = fmaxf(m, sm[w]);
  l = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = 0.f;
  for (int w = 0; w < kJoinWarps; ++w) {
    const float f = exp2_fast(sm[w] - m);
    l = fmaf(f, sl[w], l);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = fmaf(f, sy[w][4 * lane + e], y[e]);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] *= inv;
  if (v.rotate) {
    wht_32x4(y, lane);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = __uint_as_float(__float_as_uint(y[e] * 0.0625f) ^ sign_flip(v, 4 * lane + e));
  }
  const Group grp = group_of<SEL>(a, d.x);
  const int h = SEL ? grp.h : d.y / a.n_blocks, t = SEL ? grp.t : row / v.G, g = SEL ? row : row % v.G;
  uint16_t* o = a.out + grp.b * a.ob + t * a.ot + (int64_t)(h * v.G + g) * a.oh + 4 * lane;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = float_to_row(y[e], v.half);
  if (a.lse && lane == 0)
    a.lse[((int64_t)grp.b * a.T + t) * (v.H * v.G) + h * v.G + g] = l == 0.f ? kNegInf : (m + log2f(l)) * 0.693147180559945f;
}

// Workspace: descriptors, then slots.
constexpr size_t kShareDescBytes = (kPagedMaxGrid * sizeof(int4) + 255) & ~(size_t)255;

static_assert(sizeof(Smem<1>) <= 115712, "two CTAs of an SM share 228 KiB, 1 KiB each of it taken");
static_assert(sizeof(Smem<2>) <= 232448, "shared memory of a CTA");

template <int NG, int NT, bool HILO, bool SEL>
int launch(const AttnArgs& a, int dev, int sms, cudaStream_t stream) {
  auto* kernel = akv_paged_attn_kernel<NG, NT, HILO, SEL>;
  const size_t smem = sizeof(Smem<NT>);
  cudaError_t e;
  static std::atomic<uint64_t> ready{0};  // devices on which the kernel's shared memory has been set
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return (int)e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  int grid = sms * ctas_of(NT);
  if (grid > kPagedMaxGrid) grid = kPagedMaxGrid;
  const int err = launch_after(kernel, dim3(grid), Smem<NT>::kThreads, smem, stream, a);
  // units of one tile at most are nobody's share (100 tokens: 8.7 us a call with the second launch, 6.6 without)
  if (err || ((int64_t)(SEL ? a.top : a.v.max_pages) << a.v.page_log) <= kTileTokens) return err;
  return launch_after(akv_paged_join_kernel<SEL>, dim3(grid, a.rows < 8 * NT ? a.rows : 8 * NT), 32 * kJoinWarps, 0, stream, a, 8 * NT);
}

template <int NT, bool HILO, bool SEL>
int launch_ng(const AttnArgs& a, int dev, int sms, cudaStream_t s) {
  return a.v.ng == 2 ? launch<2, NT, HILO, SEL>(a, dev, sms, s) : launch<1, NT, HILO, SEL>(a, dev, sms, s);
}
template <bool HILO, bool SEL>
int launch_nt(const AttnArgs& a, int unit_rows, int dev, int sms, cudaStream_t s) {
  return unit_rows == 8 ? launch_ng<1, HILO, SEL>(a, dev, sms, s) : launch_ng<2, HILO, SEL>(a, dev, sms, s);
}

}  // namespace

size_t paged_attn_ws_bytes(const PagedView& v, int32_t T, int32_t top) {
  const int rows = paged_unit_rows(top > 0 ? v.G : T * v.G);
  return kShareDescBytes + kPagedMaxGrid * 2 * paged_slot_floats(rows) * sizeof(float);
}

int launch_paged_attn(const PagedView& v, const akv_rows& q, const akv_rows& out, float* lse, int32_t T, float sm_scale,
                      const akv_selection* sel, void* ws, void* stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return (int)e;
  AttnArgs a{};
  a.v = v;
  a.q = (const uint16_t*)q.ptr;
  a.qb = q.stride_b, a.qt = q.stride_t, a.qh = q.stride_h;
  a.out = (uint16_t*)out.ptr;
  a.ob = out.stride_b, a.ot = out.stride_t, a.oh = out.stride_h;
  a.lse = lse;
  a.scale = (float)((double)sm_scale * 1.4426950408889634);
  a.T = T;
  a.rows = sel ? v.G : T * v.G;
  const int unit_rows = paged_unit_rows(a.rows);
  a.n_blocks = (a.rows + unit_rows - 1) / unit_rows;
  if (sel) {
    a.sel = sel->pages;
    a.count = sel->count;
    a.top = sel->top;
    a.groups = v.rows * T * v.H;
    a.per_group = a.n_blocks;
  } else {
    a.groups = v.rows;
    a.per_group = v.H * a.n_blocks;
  }
  a.desc = (int4*)ws;
  a.slots = (float*)((uint8_t*)ws + kShareDescBytes);
  cudaStream_t s = (cudaStream_t)stream;
  if (v.rotate) return sel ? launch_nt<true, true>(a, unit_rows, dev, sms, s) : launch_nt<true, false>(a, unit_rows, dev, sms, s);
  return sel ? launch_nt<false, true>(a, unit_rows, dev, sms, s) : launch_nt<false, false>(a, unit_rows, dev, sms, s);
}

}  // namespace akv
