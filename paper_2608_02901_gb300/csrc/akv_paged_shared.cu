// Attention over pages that rows share: the shared pages once for all rows of a group, as matrix products on the fifth-generation
// tensor cores, and a launch that joins them with the rows' own tokens (akv_paged_attn.cu's part, launched before).
//
// A unit is a group's KV head and up to 128 of its query rows (members x query tokens x query heads); units are cut into tiles of
// 128 tokens, the tiles of all units into equal contiguous ranges, one per CTA, one CTA an SM.  In a CTA
//   2 warps copy codes and parameters into rings of two tiles,
//   2 x 8 warps turn them into operands, a sub-block of 16 tokens each: keys as (2 c - 15) a in two fp16 halves (the second the exact rest),
//     values as fp16(m + c a),
//   2 warps issue the products: S = Q K^T over 128 dimensions of (hi, lo) and 16 more that carry (2 m + 15 a) sum(q), so that a logit comes out
//     whole (doubled), then O += P V; Q and P come out of tensor memory, so that a product reads 4 KiB of shared memory and not 8.  (A warp goes
//     through its loop as one and elects the issuing thread at each batch: descriptors then are sums in uniform registers.  Out of a
//     loop of one thread a product took 94 to 107 cycles, where the tensor cores need 64 for 128 x 128 x 16.)
//   8 warps are the softmax: two threads a query row, half of a tile's columns each, which tell each other their largest logit:
//     p = 2^(S scale - reference), its sum, P as fp16 over S's columns.  (A thread a row, the two warpgroups' tiles in turn and the reference
//     handed from one to the other, took 243 us for 8 prompts of 32 k tokens with 8 answers each where this
//     took 219, 249 for 235 of 32 answers over 128 k.)
// What bounds it (32 answers, 8 x 8 heads, 128 k shared tokens, rotated: 200 us of 232, in all 593 TFLOP/s of the products that the formula
// has, 1420 of those that are made in the 200 us): the tensor cores work 65 % of the cycles, a warp instruction is issued in 70 %; of a
// tile's 3500 cycles the products need 2260, and the rest is the chain from S through P to the next use of its columns.  S of three tiles
// would not fit into tensor memory.  Of few rows the products cost the same.
//   S is as exact as fp32 sums: products of fp16 numbers are, a query enters as one fp16 number (a power of two times what was given)
// or, rotated, as a high and a low one.  The scales of tokens could not be applied behind the products instead: a thread that owns a row would
// read four numbers a token from shared memory, 512 bytes a warp, four times what the tensor cores need for the extra products.
//   A reference moves when a weight would pass 2^kSlack times it; a weight counts 2^kPlace in P, so that fp16 keeps 2^-11 of those
// down to 2^-19 of the reference's.  Sub-blocks with a scale above 2048 or a minimum beyond 16384 enter as 2^-5 of themselves (their
// columns of S count 32, their P is 32 times as large).  Tokens with a NaN enter as values of 0 and a NaN in S: rows that do not see
// them do not feel them.
//   Loops over a row's columns are not unrolled beyond 32: a call's first tile waits for its instructions.
#include <cuda_runtime.h>

#include <atomic>

#include "akv_device.cuh"
#include "akv_paged.cuh"
#include "akv_paged_tc.cuh"

namespace akv {
namespace {

constexpr int kRows = 128, kTile = 128;
constexpr int kSoftWarps = 8, kKeyWarps = 8, kValueWarps = 8, kMmaWarp = kSoftWarps + kKeyWarps + kValueWarps;
// Whole warpgroups, which share registers out: 28 warps of 72 at the launch, then 8 x 96 + 8 x 64 + 8 x 56 + 4 x 72.
constexpr int kThreads = 32 * (kMmaWarp + 4);
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLow = -3.402823466e38f;  // reference of a row that saw no token: below all others
constexpr float kSlack = 5.f, kPlace = 5.f;
constexpr int kMaxCtas = 256;
constexpr int kRawSub = 1024 + 256;       // codes of a sub-block's one side, and all its parameters
enum State : int8_t { kThere, kBehind, kOutside };
constexpr uint32_t kCols = 512, kColO = 256, kColQ = 384;  // tensor memory: S of two tiles, O, Q's high and low halves

struct SharedArgs {
  PagedView v;
  const uint8_t* queries;  // the query rows' records
  akv_share share;
  float* part;         // [rows][T][n_q_heads] parts, and where they are
  PagedWhere* where;
  float* slots;        // [ctas][2][kRows] parts of units that several CTAs worked on
  float scale;         // sm_scale log2(e)
  int T;
};

struct Smem {
  uint8_t k_hi[2][2 * kPanel];  // keys' high halves, which is also where a unit's queries are put together; the low ones, needed first, are
  uint8_t k_lo[2 * kPanel];     // written again while the products go on with the high ones
  uint8_t v[2][2 * kPanel];     // values: [dimension][token]
  uint8_t qx[kExtra], kx[2][kExtra];
  uint8_t raw[2][2][8 * kRawSub];  // codes and parameters as they come: keys, values; by tile modulo 2
  float row_scale[kRows], sum[2][kRows];
  float most[2][2][kRows];    // by tile modulo 2: the largest logit of each half of a row
  int lim[kRows];             // tokens of the unit that a row sees
  int64_t row_at[kRows];      // its number among all query rows; -1: none
  uint8_t big[4][8];          // sub-blocks that enter as 2^-5 of themselves, by tile modulo 4
  int8_t state[2][2][8];      // of a raw sub-block: kThere, kBehind the shared tokens, kOutside the pool
  uint64_t raw_full[2][2], raw_free[2][2];
  uint64_t k_full[2], k_free[2], lo_free, v_full[2], v_free[2], s_full[2], p_full[2], p_free[2], q_full, o_full, drained[2];
  int64_t part[kThreads / 32];
  int place[8];
  uint32_t tmem;
  int failed;
};

// A unit's share of a CTA: tiles t0 .. t0 + n - 1.
struct Segment {
  int k0, size, lead, tokens;  // the group: its first place in the order, rows, leader, shared tokens
  int h, block, tiles, t0, n;
};

struct Walk {
  int64_t lo, hi, total;
  int ctas;
};
__device__ __forceinline__ int row_in_order(const SharedArgs& a, int k) {
  const int b = a.share.order[k];
  return (uint32_t)b < (uint32_t)a.v.rows ? b : -1;
}
// The group that begins at place k of the order, and how many tiles its units have; 0: none begins here, or it is attended row by row.
__device__ __forceinline__ int group_at(const SharedArgs& a, int k, Segment& s) {
  const PagedView& v = a.v;
  const int b = row_in_order(a, k);
  if (b < 0 || a.share.leader[b] != b) return 0;
  s.k0 = k;
  s.lead = b;
  s.size = min(max(a.share.size[b], 1), v.rows - k);
  s.tokens = min(max(a.share.pages[b], 0), v.max_pages) << v.page_log;
  s.tiles = (s.tokens + kTile - 1) / kTile;
  return s.tiles;
}
__device__ __forceinline__ int blocks_of(const SharedArgs& a, const Segment& s) {
  return (int)(((int64_t)s.size * a.T * a.v.G + kRows - 1) / kRows);
}

// Every thread: the CTA's range of tiles, and its first segment.
__device__ __forceinline__ Walk plan(const SharedArgs& a, Smem& S, Segment& seg) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rows = a.v.rows;
  const int strip = (rows + kThreads - 1) / kThreads, k0 = min(rows, tid * strip), k1 = min(rows, k0 + strip);
  int64_t mine = 0;
  Segment s;
  for (int k = k0; k < k1; ++k)
    if (group_at(a, k, s)) mine += (int64_t)s.tiles * blocks_of(a, s) * a.v.H;
  int64_t inc = mine;
#pragma unroll
  for (int i = 1; i < 32; i *= 2) {
    const int64_t o = __shfl_up_sync(0xffffffffu, inc, i);
    if (lane >= i) inc += o;
  }
  if (lane == 31) S.part[warp] = inc;
  __syncthreads();
  int64_t before = inc - mine;
  Walk w;
  w.total = 0;
  for (int i = 0; i < kThreads / 32; ++i) {
    if (i < warp) before += S.part[i];
    w.total += S.part[i];
  }
  w.ctas = (int)min((int64_t)gridDim.x, w.total);
  w.lo = w.hi = 0;
  if ((int)blockIdx.x >= w.ctas) return w;
  w.lo = blockIdx.x * w.total / w.ctas;
  w.hi = (blockIdx.x + 1) * w.total / w.ctas;
  if (w.lo >= before && w.lo < before + mine) {
    int64_t rest = w.lo - before;
    for (int k = k0; k < k1; ++k) {
      if (!group_at(a, k, s)) continue;
      const int64_t here = (int64_t)s.tiles * blocks_of(a, s) * a.v.H;
      if (rest < here) break;
      rest -= here;
    }
    const int unit = (int)(rest / s.tiles), blocks = blocks_of(a, s);
    S.place[0] = s.k0, S.place[1] = unit / blocks, S.place[2] = unit % blocks, S.place[3] = (int)(rest % s.tiles);
  }
  __syncthreads();
  group_at(a, S.place[0], seg);
  seg.h = S.place[1], seg.block = S.place[2], seg.t0 = S.place[3];
  seg.n = (int)min((int64_t)(seg.tiles - seg.t0), w.hi - w.lo);
  return w;
}
// The segment after s, `left` tiles of the CTA's range still to go (> 0).
__device__ __forceinline__ void next_segment(const SharedArgs& a, Segment& s, int64_t left) {
  s.t0 = 0;
  if (++s.block == blocks_of(a, s)) {
    s.block = 0;
    if (++s.h == a.v.H) {
      s.h = 0;
      for (int k = s.k0 + 1; k < a.v.rows; ++k)
        if (group_at(a, k, s)) break;
    }
  }
  s.n = (int)min((int64_t)s.tiles, left);
}

// A unit's queries as operands, put together where the first keys will be, with what goes with its rows.  The 16 warps of both roles
// call it at each segment's start (its barriers are theirs: the first waits for the segment before), 8 rows a warp.
template <bool HILO>
__device__ __forceinline__ void build_queries(const SharedArgs& a, Smem& S, const Segment& seg, int warp) {
  const PagedView& v = a.v;
  const int lane = threadIdx.x & 31;
  constexpr int kEach = kRows / (kSoftWarps + kKeyWarps);
  static_assert(kEach == 8, "rows of place_queries");
  const int tg = a.T * v.G, rr = warp * kEach + (lane & (kEach - 1)), qi = seg.block * kRows + rr;
  const int k = seg.k0 + qi / tg, t = qi % tg / v.G, gq = qi % tg % v.G;
  const int b = k < seg.k0 + seg.size ? row_in_order(a, k) : -1;
  const int64_t row = b >= 0 ? ((int64_t)b * a.T + t) * (v.H * v.G) + seg.h * v.G + gq : -1;
  const int lim = b >= 0 ? min(seg.tokens, held_tokens(v, b) - a.T + 1 + t) : seg.tokens;
  const float down = b >= 0 ? *(const float*)(a.queries + row * kQueryRecord + 544) : 0.f;
  named_sync(2, 32 * (kSoftWarps + kKeyWarps));
  if (lane < kEach) S.lim[rr] = lim, S.row_at[rr] = row, S.row_scale[rr] = 0.5f * fabsf(a.scale) * down;  // (keys enter twice as large)
  place_queries<HILO, kEach>(
      lane, row < 0 ? nullptr : a.queries + row * kQueryRecord,
      [&](int r, int& to, uint32_t& panels, uint32_t& extra) { to = warp * kEach + r, panels = smem_u32(S.k_hi[0]), extra = smem_u32(S.qx); });
  proxy_fence();
  named_sync(2, 32 * (kSoftWarps + kKeyWarps));
}

template <int NG, bool HILO>
__global__ void __launch_bounds__(kThreads, 1) akv_paged_shared_kernel(const __grid_constant__ SharedArgs a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Smem& S = *reinterpret_cast<Smem*>(smem_raw + (1024u - (smem_u32(smem_raw) & 1023u)) % 1024u);
  constexpr uint32_t kSub = 2048 + 128 * NG;
  const PagedView& v = a.v;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  volatile int* failed = &S.failed;
  launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&S.k_full[s]), kKeyWarps);
      mbar_init(smem_u32(&S.k_free[s]), 1);
      for (int side = 0; side < 2; ++side) {
        mbar_init(smem_u32(&S.raw_full[side][s]), 1);
        mbar_init(smem_u32(&S.raw_free[side][s]), 8);
      }
      mbar_init(smem_u32(&S.v_full[s]), kValueWarps);
      mbar_init(smem_u32(&S.v_free[s]), 1);
      mbar_init(smem_u32(&S.s_full[s]), 1);
      mbar_init(smem_u32(&S.p_full[s]), kSoftWarps);
      mbar_init(smem_u32(&S.p_free[s]), 1);
      mbar_init(smem_u32(&S.drained[s]), 1);
    }
    mbar_init(smem_u32(&S.lo_free), 1);
    mbar_init(smem_u32(&S.q_full), kSoftWarps);
    mbar_init(smem_u32(&S.o_full), 1);
    S.failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // (also for the own tokens' launch, which writes nothing that is read here: what the launch before that one wrote is only sure to be seen
  // behind a wait.  Its CTAs leave no room for this one's beside them in any case; waiting takes 0 to 2 us a call.)
  wait_for_stream();
  Segment seg;
  const Walk w = plan(a, S, seg);
  if (w.lo >= w.hi) return;
  if (warp == kMmaWarp) tc_alloc(smem_u32(&S.tmem), kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, S.tmem, 0);

  if (warp >= kMmaWarp) {
    // (72 registers, as launched)
    if (warp < kMmaWarp + 2) {
      // ---- the products: S = Q K^T by one warp, O += P V by another, so that neither waits while the other's could run
      constexpr uint32_t idesc = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);  // fp16 x fp16 -> fp32, 128 x 128
      // D (+)= A B^T over 128 of K, A out of tensor memory, its second half `gap` columns further on
      auto product = [&](uint32_t d, uint32_t at, uint32_t gap, uint64_t desc, bool first) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          tc_mma_ts(d, at + 8 * kk + (kk >> 2) * gap, desc + (((uint32_t)(kk >> 2) * kPanel + (uint32_t)(kk & 3) * 32) >> 4), idesc, !first || kk > 0);
      };
      uint32_t n = 0, nseg = 0;
      bool ok = true;
      if (warp == kMmaWarp) {
        const uint64_t dqx = plain_desc(smem_u32(S.qx));
        for (int64_t at = w.lo; ok && at < w.hi; ++nseg) {
          ok = mbar_wait_w(smem_u32(&S.q_full), nseg & 1);
#pragma unroll 1
          for (int i = 0; ok && i < seg.n; ++i, ++n) {
            // (P of the tile two before lies over this one's S)
            const uint32_t s = n & 1;
            ok = mbar_wait_w(smem_u32(&S.k_full[s]), n >> 1 & 1) && (n < 2 || mbar_wait_w(smem_u32(&S.p_free[s]), (n - 2) >> 1 & 1)) && !warp_failed(failed);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              const uint32_t d = tmem + 128 * s;
              const uint64_t dk = sw128_desc(smem_u32(S.k_hi[s]));
              product(d, tmem + kColQ, 0, sw128_desc(smem_u32(S.k_lo)), true);
              tc_commit(smem_u32(&S.lo_free));
              if (HILO) product(d, tmem + kColQ + 64, 0, dk, false);
              product(d, tmem + kColQ, 0, dk, false);
              tc_mma(d, dqx, plain_desc(smem_u32(S.kx[s])), idesc, 1);
              tc_commit(smem_u32(&S.k_free[s]));
              tc_commit(smem_u32(&S.s_full[s]));
            }
            __syncwarp();
          }
          at += seg.n;
          if (at < w.hi) next_segment(a, seg, w.hi - at);
        }
      } else {
        for (int64_t at = w.lo; ok && at < w.hi; ++nseg) {
#pragma unroll 1
          for (int i = 0; ok && i < seg.n; ++i, ++n) {
            const uint32_t s = n & 1;
            ok = mbar_wait_w(smem_u32(&S.v_full[s]), n >> 1 & 1) && mbar_wait_w(smem_u32(&S.p_full[s]), n >> 1 & 1) && !warp_failed(failed);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              product(tmem + kColO, tmem + 128 * s, 32, sw128_desc(smem_u32(S.v[s])), i == 0);
              tc_commit(smem_u32(&S.v_free[s]));
              tc_commit(smem_u32(&S.p_free[s]));
              if (i + 1 == seg.n) tc_commit(smem_u32(&S.o_full));
            }
            __syncwarp();
          }
          at += seg.n;
          if (at < w.hi) next_segment(a, seg, w.hi - at);
        }
      }
      if (!ok) *failed = 1;
      const uint32_t drained = smem_u32(&S.drained[warp - kMmaWarp]);
      if (elect_one()) tc_commit(drained);
      __syncwarp();
      mbar_wait_w(drained, 0);  // nothing is under way when tensor memory is given back
    } else {
      // ---- copies of keys, and of values: a warp each, a lane a sub-block; the table's page numbers are looked up two tiles before
      const int side = warp - kMmaWarp - 2;
      asm volatile("fence.proxy.async.global;" ::: "memory");  // (what launches before this one wrote with ordinary stores)
      uint32_t n = 0;
      auto look = [&](int t) {  // page of the lane's sub-block of the unit's tile t: as the table says, behind the shared tokens INT32_MIN
        const int tok = t * kTile + 16 * lane;
        return lane < 8 && tok < seg.tokens ? v.table[(int64_t)seg.lead * v.table_stride + (tok >> v.page_log)] : INT32_MIN;
      };
      bool ok = true;
      for (int64_t at = w.lo; ok && at < w.hi;) {
        int page = look(seg.t0), next = look(seg.t0 + 1);
#pragma unroll 1
        for (int i = 0; i < seg.n; ++i, ++n) {
          const int t = seg.t0 + i, tok = t * kTile + 16 * lane, after = look(t + 2);
          const uint32_t st = n & 1;
          const bool there = (uint32_t)page < (uint32_t)v.n_pages;
          const uint32_t copies = __popc(__ballot_sync(0xffffffffu, there));
          ok = mbar_wait_w(smem_u32(&S.raw_free[side][st]), (n >> 1 & 1) ^ 1) && !warp_failed(failed);
          if (!ok) break;
          if (lane < 8) S.state[side][st][lane] = there ? kThere : page == INT32_MIN ? kBehind : kOutside;
          __syncwarp();
          const uint32_t bar = smem_u32(&S.raw_full[side][st]), to = smem_u32(&S.raw[side][st][lane * kRawSub]);
          if (lane == 0) mbar_expect_tx(bar, copies * (1024 + 128 * NG));
          __syncwarp();
          if (there) {
            const uint8_t* from = block_of(v, page, seg.h) + (uint64_t)((tok & ((1 << v.page_log) - 1)) >> 4) * kSub;
            bulk_g2s(to, from + 1024 * side, 1024, bar);
            bulk_g2s(to + 1024, from + 2048, 128 * NG, bar);
          }
          page = next, next = after;
        }
        at += seg.n;
        if (at < w.hi) next_segment(a, seg, w.hi - at);
      }
      if (!ok) *failed = 1;
      // shared memory is the copies' until the last have landed, also where somebody has given up
      for (uint32_t k = n > 2 ? n - 2 : 0; k < n; ++k) mbar_wait_w(smem_u32(&S.raw_full[side][k & 1]), k >> 1 & 1);
    }
  } else if (warp >= kSoftWarps) {
    // ---- operands of keys, and of values: a sub-block a warp of each
    const bool keys = warp < kSoftWarps + kKeyWarps;
    const int side = keys ? 0 : 1, u = (warp - kSoftWarps) & 7, quad = lane >> 2, t4 = lane & 3;
    uint4 c[2];            // codes
    uint32_t pw[2 * NG];   // all words of token lane % 16
    // Tokens behind the end are zeros, those of pages outside the pool have NaN parameters.
    auto load = [&](uint32_t n) {
      const uint32_t st = n & 1;
      if (!mbar_wait_w(smem_u32(&S.raw_full[side][st]), n >> 1 & 1) || warp_failed(failed)) return false;
      const int state = *(volatile int8_t*)&S.state[side][st][u];
      const uint8_t* b = &S.raw[side][st][u * kRawSub];
      c[0] = *(const uint4*)(b + 16 * lane), c[1] = *(const uint4*)(b + 512 + 16 * lane);
      if (NG == 2) {
        const uint4 x = *(const uint4*)(b + 1024 + 16 * (lane & 15));
        pw[0] = x.x, pw[1] = x.y, pw[2 * NG - 2] = x.z, pw[2 * NG - 1] = x.w;
      } else {
        const uint2 x = *(const uint2*)(b + 1024 + 8 * (lane & 15));
        pw[0] = x.x, pw[1] = x.y;
      }
      if (state != kThere) {
        c[0] = c[1] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int x = 0; x < 2 * NG; ++x) pw[x] = state == kBehind ? 0u : 0x7e007e00u;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&S.raw_free[side][st]));
      return true;
    };
    // The sub-block's size (scales beyond 2048, minima beyond 16384), and whether the token is without an infinity or a NaN
    auto look = [&](bool& fine) {
      uint32_t most = pw[0] & 0x7fff7fffu;
#pragma unroll
      for (int x = 1; x < 2 * NG; ++x) most = bits(__hmax2_nan(as_half2(most), as_half2(pw[x] & 0x7fff7fffu)));
      fine = (most & 0xffffu) < 0x7c00u && most < 0x7c000000u;
      return (bool)__any_sync(0xffffffffu, fine && ((most & 0xffffu) > 0x6800u || most > 0x7400ffffu));
    };
    uint32_t n_tile = 0, nseg = 0;
    bool ok = true;
    if (keys) {
      fewer_registers<64>();
      // tokens lane / 4 and 8 more, dimensions 32 j + 8 t + i with t = lane % 4
      const uint32_t kx_at = smem_u32(S.kx[0]) + extra_at(16 * u + (lane & 15));
      const uint32_t k_at = (uint32_t)(16 * u + quad) * 128;
      const KeyCodes codes;
      for (int64_t at = w.lo; at < w.hi; ++nseg) {
        build_queries<HILO>(a, S, seg, warp);
        // (the queries were put together in a key operand's place)
        ok = ok && mbar_wait_w(smem_u32(&S.q_full), nseg & 1);
#pragma unroll 1
        for (int i = 0; ok && i < seg.n; ++i, ++n_tile) {
          const uint32_t s = n_tile & 1, unused = (n_tile >> 1 & 1) ^ 1, hi_row = smem_u32(S.k_hi[s]) + k_at, lo_up = smem_u32(S.k_lo) - smem_u32(S.k_hi[s]);
          ok = load(n_tile);
          if (!ok) break;
          bool fine;
          const bool big = look(fine);
          const float down = big ? kLargeDown : 1.f;
          uint32_t words[NG], both[2][NG];  // of token lane % 16; of tokens lane / 4 and 8 more
#pragma unroll
          for (int x = 0; x < NG; ++x) {
            words[x] = fine ? pw[x] : 0u;
#pragma unroll
            for (int r = 0; r < 2; ++r) both[r][x] = __shfl_sync(0xffffffffu, words[x], quad + 8 * r);
          }
          ok = mbar_wait_w(smem_u32(&S.k_free[s]), unused) && mbar_wait_w(smem_u32(&S.lo_free), (n_tile & 1) ^ 1);
          if (!ok) break;
          if (lane == 0) S.big[n_tile & 3][u] = big;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            __half2 scale[NG];
#pragma unroll
            for (int x = 0; x < NG; ++x) scale[x] = __hmul2(__half2half2(__ushort_as_half((unsigned short)both[r][x])), __float2half2_rn(down));
            // (odd tokens take their words in another order: then eight lanes write eight places)
            const bool odd = quad & 1;
            const uint32_t to_r = hi_row + 1024 * r + 16 * ((odd ? 4 + t4 : t4) ^ (quad & 7));
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
              const uint32_t even_word = jj == 0 ? c[r].x : jj == 1 ? c[r].y : jj == 2 ? c[r].z : c[r].w;
              const uint32_t odd_word = jj == 0 ? c[r].y : jj == 1 ? c[r].x : jj == 2 ? c[r].w : c[r].z;
              uint32_t hi[4], lo[4];
              key_word(codes, odd ? odd_word : even_word, scale[NG == 2 ? jj >> 1 : 0], hi, lo);
              const uint32_t to = (to_r ^ (jj & 1 ? 64u : 0u)) + (uint32_t)(jj >> 1) * kPanel;
              sts128(to, make_uint4(hi[0], hi[1], hi[2], hi[3]));
              sts128(to + lo_up, make_uint4(lo[0], lo[1], lo[2], lo[3]));
            }
          }
          if (lane < 16) {
            uint4 first, second;
            key_extra<NG>(words, down, !fine, 0.f, first, second);
            sts128(kx_at + s * kExtra, first);
            sts128(kx_at + s * kExtra + 2048, second);
          }
          proxy_fence();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&S.k_full[s]));
        }
        at += seg.n;
        if (at < w.hi) next_segment(a, seg, w.hi - at);
      }
    } else {
      // tokens 2 t, 2 t + 1 of each 8 with t = lane % 4 and, after an exchange among four lanes, all 8 of dimensions 64 s + 8 g + 4 u + n with
      // g = lane / 4, 2 s + u = lane % 4
      fewer_registers<56>();
      const ValueCodes codes;
      const uint32_t tiles = (uint32_t)(w.hi - w.lo);
#pragma unroll 1
      for (; n_tile < tiles; ++n_tile) {
        ok = load(n_tile);
        if (!ok) break;
        bool fine;
        const __half2 down = __float2half2_rn(look(fine) ? kLargeDown : 1.f);
        // scales and minima in pairs of tokens: lanes 16 g + 2 x have tokens 2 x, 2 x + 1 and group g (of one group all have it)
        const uint32_t mine = fine ? NG == 2 && lane >= 16 ? pw[2 * NG - 1] : pw[NG] : 0u, next = __shfl_xor_sync(0xffffffffu, mine, 1);
        const uint32_t pair_a = bits(__hmul2(as_half2(__byte_perm(mine, next, 0x5410)), down));
        const uint32_t pair_m = bits(__hmul2(as_half2(__byte_perm(mine, next, 0x7632)), down));
        ok = mbar_wait_w(smem_u32(&S.v_free[n_tile & 1]), (n_tile >> 1 & 1) ^ 1);
        if (!ok) break;
        // dimension 64 s + 8 g + 4 u + n is operand row 32 n + 4 g + 2 s + u: eight lanes write eight places
        const uint32_t v_to = smem_u32(S.v[n_tile & 1]) + (uint32_t)(u >> 2) * kPanel + 128 * lane;
        const bool odd = t4 & 1, high = t4 & 2;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          // word lane % 4 of tokens 2 t, 2 t + 1, t = 0 .. 3
          const uint32_t r0 = __shfl_xor_sync(0xffffffffu, odd ? c[p].x : c[p].y, 1), r1 = __shfl_xor_sync(0xffffffffu, odd ? c[p].z : c[p].w, 1);
          const uint32_t a0 = odd ? r0 : c[p].x, a1 = odd ? c[p].y : r0, b0 = odd ? r1 : c[p].z, b1 = odd ? c[p].w : r1;
          const uint32_t r2 = __shfl_xor_sync(0xffffffffu, high ? a0 : b0, 2), r3 = __shfl_xor_sync(0xffffffffu, high ? a1 : b1, 2);
          const uint32_t x[4] = {high ? r2 : a0, high ? r3 : a1, high ? b0 : r2, high ? b1 : r3};
          __half2 sc[4], mn[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int from = 8 * p + 2 * t + (high ? 16 : 0);  // (dimensions 64 s .. are group s of two)
            sc[t] = as_half2(__shfl_sync(0xffffffffu, pair_a, from));
            mn[t] = as_half2(__shfl_sync(0xffffffffu, pair_m, from));
          }
          const uint32_t to = v_to + 16 * ((2 * (u & 3) + p) ^ (lane & 7));
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            // (nibbles n and n + 4 are the two tokens)
            uint32_t z[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) z[t] = bits(__hfma2(codes(x[t], x[t] >> 8, n), sc[t], mn[t]));
            sts128(to + 4096 * n, make_uint4(z[0], z[1], z[2], z[3]));
          }
        }
        proxy_fence();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.v_full[n_tile & 1]));
      }
    }
    if (!ok) *failed = 1;
  } else {
    // ---- softmax: two threads a query row, half of a tile's columns each
    more_registers<96>();
    const int half = warp >> 2, quarter = warp & 3, row = tid & 127;
    const uint32_t lane_at = tmem + ((uint32_t)(quarter * 32) << 16);
    uint32_t nseg = 0, n_tile = 0;
    for (int64_t at = w.lo; at < w.hi; ++nseg) {
      build_queries<HILO>(a, S, seg, warp);
      // a thread takes its row's high or low halves into tensor memory
      if (half == 0 || HILO)
#pragma unroll 1
        for (int p = 0; p < 2; ++p) {
          float x[32];
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const float4 y = *(const float4*)(S.k_hi[0] + (2 * half + p) * kPanel + 128 * row + 16 * (c ^ (row & 7)));
            x[4 * c] = y.x, x[4 * c + 1] = y.y, x[4 * c + 2] = y.z, x[4 * c + 3] = y.w;
          }
          tm_st32(lane_at + kColQ + 64 * half + 32 * p, x);
        }
      tm_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&S.q_full));


      const bool idle = __all_sync(0xffffffffu, S.row_at[row] < 0);  // (what P holds in these rows stays in them)
      const float row_scale = S.row_scale[row];
      const int lim = S.lim[row] - seg.t0 * kTile;  // from the segment's first token
      float ref = kLow;
      float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
      for (int i = 0; i < seg.n; ++i) {
        const uint32_t n = n_tile + i, s = n & 1, tS = lane_at + 128 * s + 64 * half;
        // (after a failure the loop goes on without waiting: two warps meet in it)
        if (warp_failed(failed) || !mbar_wait_w(smem_u32(&S.s_full[s]), n >> 1 & 1)) *failed = 1;
        if (idle) {
          if (lane == 0) mbar_arrive(smem_u32(&S.p_full[s]));
          continue;
        }
        tc_fence_after();
        const int sees = lim - i * kTile - 64 * half;
        const uint32_t big = *(const volatile uint32_t*)&S.big[n & 3][4 * half];
        // tiles that every row sees whole, without large sub-blocks, are what there is most of
        const bool plain = __all_sync(0xffffffffu, sees >= 64 && big == 0);
        // the largest logit
        float most = kNegInf;
        if (plain) {
          float m4[4] = {kNegInf, kNegInf, kNegInf, kNegInf};
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            float x[32];
            tm_ld32(tS + 32 * c, x);
#pragma unroll
            for (int e = 0; e < 32; e += 2) m4[e >> 1 & 3] = max3(m4[e >> 1 & 3], x[e], x[e + 1]);
          }
          most = fmaxf(max3(m4[0], m4[1], m4[2]), m4[3]);
        } else {
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            float x[32], m2[2] = {kNegInf, kNegInf};
            tm_ld32(tS + 32 * c, x);
#pragma unroll
            for (int e = 0; e < 32; ++e) m2[e >> 4] = fmaxf(m2[e >> 4], 32 * c + e < sees ? x[e] : kNegInf);
#pragma unroll
            for (int y = 0; y < 2; ++y) most = fmaxf(most, big >> (8 * (2 * c + y)) & 1 ? 32.f * m2[y] : m2[y]);
          }
        }
        most *= row_scale;
        *(volatile float*)&S.most[s][half][row] = most;
        named_sync(3 + quarter, 64);  // (1 and 2 are the barriers of all softmax warps, and of those with the key warps)
        most = fmaxf(most, *(volatile float*)&S.most[s][half ^ 1][row]);
        const bool up = most - ref > kSlack;  // (a row that sees nothing here sees nothing later)
        if (__any_sync(0xffffffffu, up)) {
          const float to = up ? most : ref, f = up ? exp2_fast(ref - to) : 1.f;
          ref = to;
#pragma unroll
          for (int e = 0; e < 2; ++e) sum[e].x *= f, sum[e].y *= f;
          if (i) {  // O, once the tile before is in it
            if (warp_failed(failed) || !mbar_wait_w(smem_u32(&S.v_free[s ^ 1]), (n - 1) >> 1 & 1)) *failed = 1;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {
              float x[32];
              tm_ld32(lane_at + kColO + 64 * half + 32 * c, x);
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] *= f;
              tm_st32(lane_at + kColO + 64 * half + 32 * c, x);
            }
            tm_wait_st();
          }
        }
        const float shift = kPlace - ref;
        if (plain) {
          const float2 sc = make_float2(row_scale, row_scale), sh = make_float2(shift, shift);
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            float x[32];
            tm_ld32(tS + 32 * c, x);
            uint32_t pk[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float2 y = __ffma2_rn(make_float2(x[2 * e], x[2 * e + 1]), sc, sh);
              y.x = exp2_fast(y.x), y.y = exp2_fast(y.y);
              sum[e & 1] = __fadd2_rn(sum[e & 1], y);
              pk[e] = half2_bits(y.x, y.y);
            }
            tm_st16(tS + 16 * c, pk);
          }
        } else {
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            float x[32];
            tm_ld32(tS + 32 * c, x);
            uint32_t pk[16];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const bool b = big >> (8 * (2 * c + y)) & 1;
              const float sc = b ? 32.f * row_scale : row_scale;
#pragma unroll
              for (int e = 16 * y; e < 16 * y + 16; ++e) {
                x[e] = 32 * c + e < sees ? exp2_fast(fmaf(x[e], sc, shift)) : 0.f;
                if (e & 1) sum[e >> 1 & 1].y += x[e];
                else sum[e >> 1 & 1].x += x[e];
                if (b) x[e] *= 32.f;
              }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) pk[e] = half2_bits(x[2 * e], x[2 * e + 1]);
            tm_st16(tS + 16 * c, pk);
          }
        }
        tm_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.p_full[s]));
      }
      n_tile += seg.n;
      // ---- the segment's end: each half of the threads takes half of the columns
      const bool done = !warp_failed(failed) && mbar_wait_w(smem_u32(&S.o_full), nseg & 1);
      if (!done) *failed = 1;
      S.sum[half][row] = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      named_sync(1, 32 * kSoftWarps);
      tc_fence_after();
      const bool whole = seg.t0 == 0 && seg.n == seg.tiles;
      const int64_t out_row = S.row_at[row];
      float* to = whole ? a.part + (out_row < 0 ? 0 : out_row) * kPartFloats
                        : a.slots + ((size_t)(2 * blockIdx.x + (seg.t0 == 0)) * kRows + row) * kPartFloats;
      if (!idle)
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          float x[32];
          tm_ld32(lane_at + kColO + 64 * half + 32 * c, x);
          if (out_row >= 0) {
            // (in the operand's order: the join puts it right)
#pragma unroll
            for (int e = 0; e < 32; e += 4) *(float4*)(to + 64 * half + 32 * c + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
          }
        }
      if (half == 0 && out_row >= 0) {
        const float l = S.sum[0][row] + S.sum[1][row];
        to[kD] = l == 0.f ? kLow : ref - kPlace;
        to[kD + 1] = done ? l : __int_as_float(0x7fffffff);
        if (seg.t0 == 0) {
          const int64_t last = at + seg.tiles - 1;
          const int at_last = (int)(((last + 1) * w.ctas - 1) / w.total);
          a.where[out_row] = PagedWhere{whole ? -1 : (int)blockIdx.x, at_last - (int)blockIdx.x + 1};
        }
      }
      tc_fence_before();
      at += seg.n;
      if (at < w.hi) next_segment(a, seg, w.hi - at);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) tc_dealloc(tmem, kCols);
}

// The parts of every query row together: its own tokens' and the shared ones', each whole or in the slots of several CTAs.  A warp a row.
struct JoinArgs {
  PagedView v;
  akv_share share;
  const float *own_part, *own_slots, *pre_part, *pre_slots;
  const PagedWhere *own_where, *pre_where;
  uint16_t* out;
  float* lse;
  int64_t ob, ot, oh, total;  // total: query rows
  int T, own_rows;            // own_rows: rows of an own slot
};
constexpr int kJoinWarps = 8;
__global__ void __launch_bounds__(32 * kJoinWarps) akv_paged_shared_join_kernel(const __grid_constant__ JoinArgs a) {
  launch_dependents();
  wait_for_stream();
  const PagedView& v = a.v;
  const int lane = threadIdx.x & 31, hq = v.H * v.G;
  const int64_t row = (int64_t)blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
  if (row >= a.total) return;
  const int64_t bt = row / hq;
  const int head = (int)(row % hq), b = (int)(bt / a.T), t = (int)(bt % a.T), g = head % v.G;
  float m = kLow, l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
  // dimensions 4 lane + n = 64 s + 8 g + 4 u + n lie at 32 n + 4 g + 2 s + u of shared parts
  const int place = 4 * (lane >> 1 & 7) + 2 * (lane >> 4) + (lane & 1);
  auto add = [&](int n, auto at, auto ml, bool shared) {  // n parts, four under way at a time
    for (int i0 = 0; i0 < n; i0 += 4) {
      float4 x[4];
      float2 s[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        x[u] = make_float4(0.f, 0.f, 0.f, 0.f), s[u] = make_float2(kLow, 0.f);
        if (i0 + u < n) {
          const float* p = at(i0 + u);
          x[u] = shared ? make_float4(p[place], p[32 + place], p[64 + place], p[96 + place]) : *(const float4*)(p + 4 * lane);
          s[u] = *(const float2*)ml(i0 + u);
        }
      }
      const float mn = fmaxf(m, fmaxf(fmaxf(s[0].x, s[1].x), fmaxf(s[2].x, s[3].x))), f = exp2_fast(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] *= f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i0 + u >= n) break;
        const float w = exp2_fast(s[u].x - m);
        l = fmaf(w, s[u].y, l);
        y[0] = fmaf(w, x[u].x, y[0]);
        y[1] = fmaf(w, x[u].y, y[1]);
        y[2] = fmaf(w, x[u].z, y[2]);
        y[3] = fmaf(w, x[u].w, y[3]);
      }
    }
  };
  // shared pages; the block of 128 that the row is in counts from its group's first row
  const int lead = a.share.leader[b];
  if ((uint32_t)lead < (uint32_t)v.rows && min(a.share.pages[lead], v.max_pages) > 0) {
    const PagedWhere w = a.pre_where[row];
    if (w.first < 0) {
      const float* p = a.pre_part + row * kPartFloats;
      add(1, [&](int) { return p; }, [&](int) { return p + kD; }, true);
    } else {
      int before = 0;  // members of the group before the row: rows with its leader and a lower number
      for (int j0 = 0; j0 < b; j0 += 32) before += __popc(__ballot_sync(0xffffffffu, j0 + lane < b && a.share.leader[j0 + lane] == lead));
      const int rr = (int)((((int64_t)before * a.T + t) * v.G + g) % kRows), first = min(w.first, kMaxCtas - 1), n = min(w.n, kMaxCtas - first);
      auto at = [&](int i) { return a.pre_slots + ((size_t)(2 * (first + i) + (i == 0)) * kRows + rr) * kPartFloats; };
      add(n, at, [&](int i) { return at(i) + kD; }, true);
    }
  }
  {
    const PagedWhere w = a.own_where[row];
    if (w.first < 0) {
      const float* p = a.own_part + row * kPartFloats;
      add(1, [&](int) { return p; }, [&](int) { return p + kD; }, false);
    } else {
      const int rr = (t * v.G + g) % a.own_rows, first = min(w.first, kPagedMaxGrid - 1), n = min(w.n, kPagedMaxGrid - first);
      auto slot = [&](int i) { return a.own_slots + (2 * (size_t)(first + i) + (i == 0)) * paged_slot_floats(a.own_rows); };
      add(n, [&](int i) { return slot(i) + rr * kD; }, [&](int i) { return slot(i) + a.own_rows * kD + 2 * rr; }, false);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] *= inv;
  if (v.rotate) {
    wht_32x4(y, lane);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = __uint_as_float(__float_as_uint(y[e] * 0.0625f) ^ sign_flip(v, 4 * lane + e));
  }
  uint16_t* o = a.out + b * a.ob + t * a.ot + (int64_t)head * a.oh + 4 * lane;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = float_to_row(y[e], v.half);
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? kNegInf : (m + log2f(l)) * 0.693147180559945f;
}

template <int NG, bool HILO>
int launch(const SharedArgs& a, int dev, int sms, void* stream) {
  auto* kernel = akv_paged_shared_kernel<NG, HILO>;
  constexpr size_t smem = sizeof(Smem) + 1024;
  static_assert(smem <= 232448, "shared memory of a CTA");
  static std::atomic<uint64_t> ready{0};  // devices on which the kernel's shared memory has been set
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return (int)e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_after(kernel, dim3(sms < kMaxCtas ? sms : kMaxCtas), kThreads, smem, stream, a);
}

// Workspace: the own part's (its slots), then parts and places of both sides, shared pages of rows, the query rows' records, the shared part's slots.
struct SharedWs {
  size_t own_part, own_where, pre_part, pre_where, shared, queries, slots, total;
};
SharedWs shared_ws(const PagedView& v, int32_t T) {
  const size_t rows = (size_t)v.rows * T * v.H * v.G;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  SharedWs w;
  w.own_part = up(paged_attn_ws_bytes(v, T, 0));
  w.own_where = w.own_part + up(rows * kPartFloats * sizeof(float));
  w.pre_part = w.own_where + up(rows * sizeof(PagedWhere));
  w.pre_where = w.pre_part + up(rows * kPartFloats * sizeof(float));
  w.shared = w.pre_where + up(rows * sizeof(PagedWhere));
  w.queries = w.shared + up((size_t)v.rows * sizeof(int32_t));
  w.slots = w.queries + up(rows * kQueryRecord);
  w.total = w.slots + (size_t)kMaxCtas * 2 * kRows * kPartFloats * sizeof(float);
  return w;
}

}  // namespace

size_t paged_shared_ws_bytes(const PagedView& v, int32_t T) { return shared_ws(v, T).total; }

int launch_paged_shared(const PagedView& v, const akv_rows& q, const akv_rows& out, float* lse, int32_t T, float sm_scale,
                        const akv_share& given, void* ws, void* stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return (int)e;
  const SharedWs w = shared_ws(v, T);
  uint8_t* base = (uint8_t*)ws;
  akv_share share = given;
  share.pages = (int32_t*)(base + w.shared);  // what of each row's pages is read once for its group
  PagedOwn own;
  own.pages = share.pages;
  own.part = (float*)(base + w.own_part);
  own.where = (PagedWhere*)(base + w.own_where);
  int err = launch_paged_queries(v, q, T, sm_scale < 0.f, nullptr, &given, share.pages, base + w.queries, stream);
  if (!err) err = launch_paged_own(v, q, T, sm_scale, own, ws, stream);
  if (err) return err;
  SharedArgs a{};
  a.v = v;
  a.queries = base + w.queries;
  a.share = share;
  a.part = (float*)(base + w.pre_part);
  a.where = (PagedWhere*)(base + w.pre_where);
  a.slots = (float*)(base + w.slots);
  a.scale = (float)((double)sm_scale * 1.4426950408889634);
  a.T = T;
  if (v.rotate) err = v.ng == 2 ? launch<2, true>(a, dev, sms, stream) : launch<1, true>(a, dev, sms, stream);
  else err = v.ng == 2 ? launch<2, false>(a, dev, sms, stream) : launch<1, false>(a, dev, sms, stream);
  if (err) return err;
  JoinArgs j{};
  j.v = v;
  j.share = share;
  j.own_part = own.part, j.own_where = own.where, j.own_slots = paged_own_slots(ws);
  j.pre_part = a.part, j.pre_where = a.where, j.pre_slots = a.slots;
  j.out = (uint16_t*)out.ptr;
  j.ob = out.stride_b, j.ot = out.stride_t, j.oh = out.stride_h;
  j.lse = lse;
  j.total = (int64_t)v.rows * T * v.H * v.G;
  j.T = T;
  j.own_rows = paged_unit_rows(T * v.G);
  return launch_after(akv_paged_shared_join_kernel, dim3((unsigned)((j.total + kJoinWarps - 1) / kJoinWarps)), 32 * kJoinWarps, 0, stream, j);
}

}  // namespace akv
