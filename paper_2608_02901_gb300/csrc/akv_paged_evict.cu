// Eviction from the paged cache by scores: which tokens a row keeps, and their move to the first places of a row.
//
// A cluster per row and KV head does all of it in one launch.  The lowest score that is kept comes from a radix select over
// (forced, score) as 32-bit keys, 11, 11 and 10 bits a pass, counts joined through distributed shared memory; the kept tokens'
// places are counted off in order, each CTA over its share of the row; then the tokens move, a sub-block of 16 a warp.
// A token's 64 bytes of key codes and its parameters are contiguous, its value codes are 32 pieces of two bytes, next to those of
// its neighbour: a warp loads the sixteen-byte units that hold them and puts two tokens' halves together (PRMT).
// In place: a kept token goes to a place at or before its own, so the places that a round of sub-blocks writes hold no token
// that a later round reads; a round is read by the whole cluster, then (cluster barrier) written.
// Bound by memory: the kept tokens' bytes, read and written, next to 4 bytes a token for the scores.
#include <cooperative_groups.h>

#include "akv_paged.cuh"

namespace cg = cooperative_groups;

namespace akv {
namespace {

constexpr int kCtas = 8, kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;

struct EvictArgs {
  PagedView v;
  const int32_t *src, *dst, *keep;
  float* scores;
  int64_t sb, sh;
  int32_t sink, recent;
  int32_t *tokens, *count;
  int32_t top;
};

// Scores in their order as whole numbers: a NaN lowest, -0 as 0; kForced above all.
constexpr uint32_t kForced = 0xffffffffu;
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint32_t smem_sum(uint32_t x, uint32_t* part) {  // over the CTA; all threads call it
  x = __reduce_add_sync(0xffffffffu, x);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  uint32_t sum = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) sum += part[w];
  return sum;
}

struct Moved {  // a warp's share of a sub-block on its way
  uint4 key[2], value[2], meta;
  float score;
};

__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads, 2) akv_paged_evict_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ uint32_t hist[kBins], slice[kBins / kCtas], part[kWarps], part2[kWarps];
  __shared__ uint32_t total, flag, n_above, n_equal, first_gone;
  cg::cluster_group cl = cg::this_cluster();
  const PagedView& v = a.v;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cl.block_rank(), unit = blockIdx.x / kCtas, pair = unit / v.H, h = unit % v.H;
  launch_dependents();
  wait_for_stream();

  // ---- what the pair is, and whether it can be done
  const int from = a.src[pair], to = a.dst[pair];
  const bool rows_ok = (uint32_t)from < (uint32_t)v.rows && (uint32_t)to < (uint32_t)v.rows;
  const int held = rows_ok ? held_tokens(v, from) : 0;
  const int m = min(held, min(max(a.keep ? a.keep[pair] : a.top, 0), a.top));
  const bool in_place = from == to, stays = in_place && m == held;
  const int P = 1 << v.page_log;
  bool bad = !rows_ok;
  for (int j = rank * kThreads + tid; j < (held + P - 1) >> v.page_log; j += kCtas * kThreads) bad = bad || page_of(v, from, j) < 0;
  for (int j = rank * kThreads + tid; j < (m + P - 1) >> v.page_log && rows_ok; j += kCtas * kThreads) {
    const int page = page_of(v, to, j);
    bad = bad || page < 0 || (!stays && v.refs && v.refs[page] > 1);
  }
  const int any_bad = __syncthreads_or(bad);
  if (tid == 0) flag = (uint32_t)any_bad, first_gone = (uint32_t)held;
  cl.sync();
  uint32_t refuse = 0;
#pragma unroll
  for (int r = 0; r < kCtas; ++r) refuse |= *cl.map_shared_rank(&flag, r);
  int32_t* list = a.tokens + (int64_t)unit * a.top;
  const int listed = refuse ? 0 : m;
  for (int k = listed + rank * kThreads + tid; k < a.top; k += kCtas * kThreads) list[k] = -1;
  if (rank == 0 && tid == 0 && h == 0) a.count[pair] = refuse ? -1 : m;
  if (refuse || m == 0) {
    cl.sync();  // (the others have read the flag)
    return;
  }

  const float* mine = a.scores + (int64_t)from * a.sb + (int64_t)h * a.sh;
  const int share = ((held + kCtas - 1) / kCtas + 31) & ~31, lo = min(held, rank * share), hi = min(held, lo + share);
  auto key_of = [&](int i) { return i < a.sink || i >= held - a.recent ? kForced : score_key(mine[i]); };

  // ---- the lowest key that is kept, and how many of that key
  uint32_t cut = 0, left = (uint32_t)m;
  if (m < held) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048, top_shift = pass == 0 ? 32 : pass == 1 ? 21 : 10;
      for (int k = tid; k < bins; k += kThreads) hist[k] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += kThreads) {
        const uint32_t k = key_of(i);
        if (pass == 0 || (k ^ cut) >> top_shift == 0) atomicAdd(&hist[k >> shift & (bins - 1)], 1u);
      }
      cl.sync();
      const int each = bins / kCtas;  // bins of a CTA
      uint32_t sum = 0;
      if (tid < each) {
#pragma unroll
        for (int r = 0; r < kCtas; ++r) sum += cl.map_shared_rank(hist, r)[rank * each + tid];
        slice[tid] = sum;
      }
      sum = smem_sum(sum, part);
      if (tid == 0) total = sum;
      cl.sync();
      int owner = kCtas - 1;  // the CTA in whose bins the count is reached, from the top
      for (; owner > 0; --owner) {
        const uint32_t there = *cl.map_shared_rank(&total, owner);
        if (there >= left) break;
        left -= there;
      }
      // thread t: bin each - 1 - t, so that sums over the threads before are sums from the top
      const uint32_t mine_n = tid < each ? cl.map_shared_rank(slice, owner)[each - 1 - tid] : 0;
      uint32_t inc = mine_n;
#pragma unroll
      for (int s = 1; s < 32; s *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, inc, s);
        if (lane >= s) inc += o;
      }
      __syncthreads();
      if (lane == 31) part[warp] = inc;
      __syncthreads();
      for (int w = 0; w < warp; ++w) inc += part[w];
      if (mine_n && inc >= left && inc - mine_n < left) part2[0] = (uint32_t)(owner * each + each - 1 - tid), part2[1] = left - (inc - mine_n);
      __syncthreads();
      cut |= part2[0] << shift;
      left = part2[1];
      cl.sync();  // (slices and histograms have been read)
    }
  }

  // ---- the list: tokens above the cut, and the first `left` at it
  uint32_t above = 0, equal = 0;
  if (m < held) {
    for (int i = lo + tid; i < hi; i += kThreads) {
      const uint32_t k = key_of(i);
      above += k > cut, equal += k == cut;
    }
    above = smem_sum(above, part);
    equal = smem_sum(equal, part);
    if (tid == 0) n_above = above, n_equal = equal;
    cl.sync();
    above = equal = 0;
    for (int r = 0; r < rank; ++r) above += *cl.map_shared_rank(&n_above, r), equal += *cl.map_shared_rank(&n_equal, r);
    constexpr int kEach = 8;  // tokens of a thread a turn
    uint32_t gone = (uint32_t)held;
    for (int i0 = lo; i0 < hi; i0 += kThreads * kEach) {
      uint32_t is_above[kEach], is_equal[kEach], na = 0, ne = 0;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = i0 + 32 * (kEach * warp + e) + lane;
        const uint32_t k = i < hi ? key_of(i) : 0;
        is_above[e] = __ballot_sync(0xffffffffu, i < hi && k > cut);
        is_equal[e] = __ballot_sync(0xffffffffu, i < hi && k == cut);
        na += __popc(is_above[e]), ne += __popc(is_equal[e]);
      }
      __syncthreads();
      if (lane == 0) part[warp] = na, part2[warp] = ne;
      __syncthreads();
      uint32_t xa = above, xe = equal;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) xa += part[w], xe += part2[w];
        above += part[w], equal += part2[w];
      }
      const uint32_t before = (1u << lane) - 1;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = i0 + 32 * (kEach * warp + e) + lane;
        const uint32_t ea = xa + __popc(is_above[e] & before), ee = xe + __popc(is_equal[e] & before);
        if ((is_above[e] >> lane & 1) || ((is_equal[e] >> lane & 1) && ee < left)) list[ea + min(ee, left)] = i;
        else if (i < hi) gone = min(gone, (uint32_t)i);
        xa += __popc(is_above[e]), xe += __popc(is_equal[e]);
      }
    }
    gone = __reduce_min_sync(0xffffffffu, gone);
    if (lane == 0) atomicMin(&first_gone, gone);
  } else {
    for (int i = lo + tid; i < hi; i += kThreads) list[i] = i;
  }
  cl.sync();  // the list is there
  int start = 0;  // tokens before the first that goes stay where they are
  if (in_place) {
    uint32_t first = (uint32_t)held;
#pragma unroll
    for (int r = 0; r < kCtas; ++r) first = min(first, *cl.map_shared_rank(&first_gone, r));
    start = (int)first >> 4;
  }
  cl.sync();  // (nobody's shared memory is read from here on)
  if (stays) return;

  // ---- the move
  const uint32_t sub_size = sub_bytes(v.ng);
  const int subs = (m + 15) >> 4;
  float* theirs = a.scores + (int64_t)to * a.sb + (int64_t)h * a.sh;
#pragma unroll 1
  for (int s0 = start; s0 < subs; s0 += kCtas * kWarps) {
    const int s = s0 + rank * kWarps + warp, n = min(16, m - 16 * s);  // tokens of the warp's sub-block
    Moved x{};
    if (n > 0) {
      // lanes 0 .. 15 look up a token each
      const int tok = __ldcg(list + 16 * s + min(lane & 15, n - 1));
      const uint8_t* base = block_of(v, page_of(v, from, tok >> v.page_log), h) + (uint64_t)((tok & (P - 1)) >> 4) * sub_size;
      auto of = [&](int k, int& place) {
        place = __shfl_sync(0xffffffffu, tok, k) & 15;
        return (const uint8_t*)__shfl_sync(0xffffffffu, (unsigned long long)base, k);
      };
      int i0, i1;
      {
        const uint8_t* b = of(lane >> 1, i0);
        const uint4* k = (const uint4*)(b + 64 * i0 + 32 * (lane & 1));
        x.key[0] = k[0], x.key[1] = k[1];
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int t = lane & 3, g = lane >> 2;
        const uint8_t *b0 = of(8 * p + 2 * t, i0), *b1 = of(8 * p + 2 * t + 1, i1);
        const uint4 y0 = *(const uint4*)(b0 + 1024 + 512 * (i0 >> 3) + 16 * (4 * g + ((i0 & 7) >> 1)));
        const uint4 y1 = *(const uint4*)(b1 + 1024 + 512 * (i1 >> 3) + 16 * (4 * g + ((i1 & 7) >> 1)));
        // the half of the first token's words, then that of the second's
        const uint32_t pick = (i0 & 1 ? 0x32u : 0x10u) | (i1 & 1 ? 0x7600u : 0x5400u);
        x.value[p] = make_uint4(__byte_perm(y0.x, y1.x, pick), __byte_perm(y0.y, y1.y, pick), __byte_perm(y0.z, y1.z, pick),
                                __byte_perm(y0.w, y1.w, pick));
      }
      if (lane < n) {
        const uint8_t* at = base + 2048 + 8 * v.ng * (tok & 15);
        if (v.ng == 2) {
          x.meta = *(const uint4*)at;
        } else {
          const uint2 w = *(const uint2*)at;
          x.meta.x = w.x, x.meta.y = w.y;
        }
        x.score = mine[tok];
      }
    }
    if (in_place) cl.sync();
    if (n > 0) {
      uint8_t* base = block_of(v, page_of(v, to, 16 * s >> v.page_log), h) + (uint64_t)((16 * s & (P - 1)) >> 4) * sub_size;
      if (lane >> 1 < n) {
        uint4* k = (uint4*)(base + 32 * lane);
        k[0] = x.key[0], k[1] = x.key[1];
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int k0 = 8 * p + 2 * (lane & 3);
        uint8_t* at = base + 1024 + 512 * p + 16 * lane;
        if (k0 + 1 < n) {
          *(uint4*)at = x.value[p];
        } else if (k0 < n) {  // the neighbour's codes stay
          uint16_t* half = (uint16_t*)at;
          half[0] = (uint16_t)x.value[p].x, half[2] = (uint16_t)x.value[p].y, half[4] = (uint16_t)x.value[p].z,
          half[6] = (uint16_t)x.value[p].w;
        }
      }
      if (lane < n) {
        uint8_t* at = base + 2048 + 8 * v.ng * lane;
        if (v.ng == 2) *(uint4*)at = x.meta;
        else *(uint2*)at = make_uint2(x.meta.x, x.meta.y);
        theirs[16 * s + lane] = x.score;
      }
    }
  }
}

}  // namespace

int launch_paged_evict(const PagedView& v, const int32_t* src, const int32_t* dst, int32_t n, const akv_scores& scores,
                       const int32_t* keep, int32_t sink, int32_t recent, const akv_kept& kept, void* stream) {
  EvictArgs a{};
  a.v = v;
  a.src = src, a.dst = dst, a.keep = keep;
  a.scores = scores.ptr;
  a.sb = scores.stride_b, a.sh = scores.stride_h;
  a.sink = sink, a.recent = recent;
  a.tokens = kept.tokens, a.count = kept.count, a.top = kept.top;
  return launch_after(akv_paged_evict_kernel, dim3((unsigned)(n * v.H * kCtas)), kThreads, 0, stream, a);
}

}  // namespace akv
