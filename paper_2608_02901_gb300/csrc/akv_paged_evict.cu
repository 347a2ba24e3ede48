// Eviction from the paged cache by scores: which tokens a row keeps, and their move to the first places of a row.
//
// A cluster per row and KV head does all of it in one launch.  The lowest score that is kept comes from a radix select over
// (forced, score) as 32-bit keys, 11, 11 and 10 bits a pass, counts joined through distributed shared memory (where the first pass leaves few keys
// open, one CTA takes them and finds the rest: a pass through the cluster is 3.5 us, 27.5 to 24.6 us of 32 k tokens cut to 4 k); the kept tokens'
// places are counted off in order, each CTA over its share of the row; then the tokens move, a sub-block of 16 a warp.
// A token's 64 bytes of key codes and its parameters are contiguous, its value codes are 32 pieces of two bytes, next to those of
// its neighbour: a warp loads the sixteen-byte units that hold them and puts two tokens' halves together (PRMT).
// In place: a kept token goes to a place at or before its own, so the places that a round of sub-blocks writes hold no token
// that a later round reads; a round is read by the whole cluster, then (cluster barrier) written.
// What bounds it: of long rows the kept tokens' bytes, read and written (4 rows of 128 k tokens, 8 heads, half of them kept, into other rows: 175 us; 640 MB
// asked for, 858 MB moved, since a 32-byte sector holds values of four tokens: 4.9 TB/s), of which a warp has one round under way at a time; in place
// each round's barrier of the cluster as well, between its reads and its writes (241 us); of short rows the chain of some twelve dependent reads and
// barriers (32 rows of 1.1 k tokens 25.9 us, in place 24.6; 32 k tokens cut to 4 k 24.8, in place 24.5).
#include <cooperative_groups.h>

#include "akv_paged.cuh"

namespace cg = cooperative_groups;

namespace akv {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kCand = 6144;  // keys that one CTA of a cluster takes
constexpr int kEach = 8, kBatch = kThreads * kEach;  // scores of a thread, of a CTA, that are under way at a time

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

// A cluster of C CTAs; one is on its own.
template <int C>
struct Cluster {
  __device__ __forceinline__ int rank() const { return C == 1 ? 0 : (int)cg::this_cluster().block_rank(); }
  __device__ __forceinline__ void sync() const {
    if (C == 1) __syncthreads();
    else cg::this_cluster().sync();
  }
  template <class T>
  __device__ __forceinline__ T* of(T* p, int r) const {
    return C == 1 ? p : cg::this_cluster().map_shared_rank(p, r);
  }
};

template <int C>
__global__ void __launch_bounds__(kThreads, 2) akv_paged_evict_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ uint32_t hist[kBins], slice[kBins / C], part[kWarps], part2[kWarps];
  __shared__ uint32_t total, flag, n_above, n_equal, first_gone, n_cand;
  __shared__ uint32_t cand[C > 1 ? kCand : 1];
  const Cluster<C> cl;
  const PagedView& v = a.v;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = cl.rank(), unit = blockIdx.x / C, pair = unit / v.H, h = unit % v.H;
  launch_dependents();
  wait_for_stream();

  // ---- what the pair is, and whether it can be done
  const int from = a.src[pair], to = a.dst[pair];
  const bool rows_ok = (uint32_t)from < (uint32_t)v.rows && (uint32_t)to < (uint32_t)v.rows;
  const int held = rows_ok ? held_tokens(v, from) : 0;
  const int m = min(held, min(max(a.keep ? a.keep[pair] : a.top, 0), a.top));
  const bool in_place = from == to, stays = in_place && m == held;
  const int P = 1 << v.page_log;

  // the CTA's share of the scores: its only batch stays in registers
  const float* mine = rows_ok ? a.scores + (int64_t)from * a.sb + (int64_t)h * a.sh : a.scores;
  const int share = ((held + C - 1) / C + 31) & ~31, lo = min(held, rank * share), hi = min(held, lo + share);
  uint32_t key[kEach];  // of tokens i0 + 32 (kEach warp + e) + lane, 0 behind the share
  auto place = [&](int i0, int e) { return i0 + 32 * (kEach * warp + e) + lane; };
  auto load = [&](int i0) {
    float x[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) x[e] = place(i0, e) < hi ? mine[place(i0, e)] : 0.f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = place(i0, e);
      key[e] = i < a.sink || i >= held - a.recent ? kForced : score_key(x[e]);
    }
  };
  auto each_batch = [&](auto f) {
    for (int i0 = lo; i0 < hi; i0 += kBatch) {
      if (hi - lo > kBatch) load(i0);
      f(i0);
    }
  };
  if (m < held && hi - lo <= kBatch) load(lo);

  bool bad = !rows_ok;
  for (int j = rank * kThreads + tid; j < (held + P - 1) >> v.page_log; j += C * kThreads) bad = bad || page_of(v, from, j) < 0;
  for (int j = rank * kThreads + tid; j < (m + P - 1) >> v.page_log && rows_ok; j += C * kThreads) {
    const int page = page_of(v, to, j);
    bad = bad || page < 0 || (!stays && v.refs && v.refs[page] > 1);
  }
  const int any_bad = __syncthreads_or(bad);
  if (tid == 0) flag = (uint32_t)any_bad, first_gone = (uint32_t)held, n_cand = 0;
  cl.sync();
  uint32_t refuse = 0;
#pragma unroll
  for (int r = 0; r < C; ++r) refuse |= *cl.of(&flag, r);
  int32_t* list = a.tokens + (int64_t)unit * a.top;
  const int listed = refuse ? 0 : m;
  for (int k = listed + rank * kThreads + tid; k < a.top; k += C * kThreads) list[k] = -1;
  if (rank == 0 && tid == 0 && h == 0) a.count[pair] = refuse ? -1 : m;
  if (refuse || m == 0) {
    cl.sync();  // (the others have read the flag)
    return;
  }

  // ---- the lowest key that is kept, and how many of that key
  uint32_t cut = 0, left = (uint32_t)m;
  if (m < held) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048, top_shift = pass == 1 ? 21 : 10;
      for (int k = tid; k < bins; k += kThreads) hist[k] = 0;
      __syncthreads();
      each_batch([&](int i0) {
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          if (place(i0, e) < hi && (pass == 0 || (key[e] ^ cut) >> top_shift == 0)) atomicAdd(&hist[key[e] >> shift & (bins - 1)], 1u);
      });
      cl.sync();
      const int each = bins / C;  // bins of a CTA
      uint32_t sum = 0;
      if (C > 1) {
        for (int k = tid; k < each; k += kThreads) {
          uint32_t x = 0;
#pragma unroll
          for (int r = 0; r < C; ++r) x += cl.of(hist, r)[rank * each + k];
          slice[k] = x;
          sum += x;
        }
        sum = smem_sum(sum, part);
        if (tid == 0) total = sum;
        cl.sync();
      }
      int owner = C - 1;  // the CTA in whose bins the count is reached, from the top
      for (; owner > 0; --owner) {
        const uint32_t there = *cl.of(&total, owner);
        if (there >= left) break;
        left -= there;
      }
      // thread t: bins each - 1 - n t and the n - 1 before, so that sums over the threads before are sums from the top
      constexpr int kMost = kBins / C > kThreads ? kBins / C / kThreads : 1;
      const int n = each > kThreads ? each / kThreads : 1;
      const uint32_t* bin = C > 1 ? cl.of(slice, owner) : hist;
      uint32_t here[kMost], inc = 0;
#pragma unroll
      for (int k = 0; k < kMost; ++k) {
        const int x = each - 1 - (n * tid + k);
        here[k] = k < n && x >= 0 ? bin[x] : 0;
        inc += here[k];
      }
      const uint32_t mine_n = inc;
#pragma unroll
      for (int s = 1; s < 32; s *= 2) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, inc, s);
        if (lane >= s) inc += o;
      }
      __syncthreads();
      if (lane == 31) part[warp] = inc;
      __syncthreads();
      for (int w = 0; w < warp; ++w) inc += part[w];
      inc -= mine_n;
#pragma unroll
      for (int k = 0; k < kMost; ++k) {
        if (here[k] && inc < left && inc + here[k] >= left) part2[0] = (uint32_t)(owner * each + each - 1 - (n * tid + k)), part2[1] = left - inc, part2[2] = here[k];
        inc += here[k];
      }
      __syncthreads();
      cut |= part2[0] << shift;
      left = part2[1];
      cl.sync();  // (slices and histograms have been read)
      if constexpr (C > 1) {
        // the keys that the first bits leave open go to one CTA, which finds the rest by itself
        if (pass == 0 && part2[2] <= (uint32_t)kCand) {
          uint32_t* const all = cl.of(cand, 0);
          each_batch([&](int i0) {
            uint32_t open[kEach], n = 0, at = 0;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
              open[e] = __ballot_sync(0xffffffffu, place(i0, e) < hi && key[e] >> 21 == cut >> 21);
              n += __popc(open[e]);
            }
            if (!n) return;
            if (lane == 0) at = atomicAdd(cl.of(&n_cand, 0), n);
            at = __shfl_sync(0xffffffffu, at, 0);
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
              if (open[e] >> lane & 1) all[at + __popc(open[e] & ((1u << lane) - 1))] = key[e];
              at += __popc(open[e]);
            }
          });
          cl.sync();
          if (rank == 0) {
            const int n = (int)part2[2];
#pragma unroll 1
            for (int low = 14; low >= 0; low -= 7) {
              if (tid < 128) hist[tid] = 0;
              __syncthreads();
              for (int k = tid; k < n; k += kThreads)
                if ((cand[k] ^ cut) >> (low + 7) == 0) atomicAdd(&hist[cand[k] >> low & 127], 1u);
              __syncthreads();
              uint32_t there[4], sum4 = 0;  // every warp: lane t bins 127 - 4 t and the three before
#pragma unroll
              for (int k = 0; k < 4; ++k) there[k] = hist[127 - 4 * lane - k], sum4 += there[k];
              uint32_t from_top = sum4;
#pragma unroll
              for (int s = 1; s < 32; s *= 2) {
                const uint32_t o = __shfl_up_sync(0xffffffffu, from_top, s);
                if (lane >= s) from_top += o;
              }
              from_top -= sum4;
              uint32_t found = 0, rest = 0;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if (there[k] && from_top < left && from_top + there[k] >= left) found = 127 - 4 * lane - k, rest = left - from_top;
                from_top += there[k];
              }
              cut |= __reduce_max_sync(0xffffffffu, found) << low, left = __reduce_max_sync(0xffffffffu, rest);
              __syncthreads();
            }
            if (tid == 0) part2[0] = cut, part2[1] = left;
          }
          cl.sync();
          cut = *cl.of(&part2[0], 0), left = *cl.of(&part2[1], 0);
          break;
        }
      }
    }
  }

  // ---- the list: tokens above the cut, and the first `left` at it
  if (m < held) {
    uint32_t above = 0, equal = 0;
    if (C > 1) {
      each_batch([&](int i0) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const bool in = place(i0, e) < hi;
          above += in && key[e] > cut, equal += in && key[e] == cut;
        }
      });
      above = smem_sum(above, part);
      equal = smem_sum(equal, part);
      if (tid == 0) n_above = above, n_equal = equal;
      cl.sync();
      above = equal = 0;
      for (int r = 0; r < rank; ++r) above += *cl.of(&n_above, r), equal += *cl.of(&n_equal, r);
    }
    uint32_t gone = (uint32_t)held;
    each_batch([&](int i0) {
      uint32_t is_above[kEach], is_equal[kEach], na = 0, ne = 0;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const bool in = place(i0, e) < hi;
        is_above[e] = __ballot_sync(0xffffffffu, in && key[e] > cut);
        is_equal[e] = __ballot_sync(0xffffffffu, in && key[e] == cut);
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
        const int i = place(i0, e);
        const uint32_t ea = xa + __popc(is_above[e] & before), ee = xe + __popc(is_equal[e] & before);
        if ((is_above[e] >> lane & 1) || ((is_equal[e] >> lane & 1) && ee < left)) list[ea + min(ee, left)] = i;
        else if (i < hi) gone = min(gone, (uint32_t)i);
        xa += __popc(is_above[e]), xe += __popc(is_equal[e]);
      }
    });
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
    for (int r = 0; r < C; ++r) first = min(first, *cl.of(&first_gone, r));
    start = (int)first >> 4;
  }
  cl.sync();  // (nobody's shared memory is read from here on)
  if (stays) return;

  // ---- the move
  const uint32_t sub_size = sub_bytes(v.ng);
  const int subs = (m + 15) >> 4;
  constexpr int kStep = C * kWarps;
  float* theirs = a.scores + (int64_t)to * a.sb + (int64_t)h * a.sh;
  // Lanes 0 .. 15 look up a token each; places two rounds ahead, pages one.
  auto token_at = [&](int s) { return s < subs ? __ldcg(list + min(16 * s + (lane & 15), m - 1)) : 0; };
  auto source_of = [&](int tok) {
    return block_of(v, page_of(v, from, tok >> v.page_log), h) + (uint64_t)((tok & (P - 1)) >> 4) * sub_size;
  };
  auto target_page = [&](int s) { return page_of(v, to, s < subs ? 16 * s >> v.page_log : 0); };
  const int first_sub = start + rank * kWarps + warp;
  int tok = token_at(first_sub), next_tok = token_at(first_sub + kStep);
  const uint8_t* source = source_of(tok);
  int page = target_page(first_sub);
#pragma unroll 1
  for (int s0 = start; s0 < subs; s0 += kStep) {
    const int s = s0 + rank * kWarps + warp, n = min(16, m - 16 * s);  // tokens of the warp's sub-block
    const uint8_t* next_source = source_of(next_tok);
    const int next_page = target_page(s + kStep);
    const int after_tok = token_at(s + 2 * kStep);
    Moved x{};
    if (n > 0) {
      auto of = [&](int k, int& at) {
        at = __shfl_sync(0xffffffffu, tok, k) & 15;
        return (const uint8_t*)__shfl_sync(0xffffffffu, (unsigned long long)source, k);
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
        const uint8_t* at = source + 2048 + 8 * v.ng * (tok & 15);
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
      uint8_t* base = block_of(v, page, h) + (uint64_t)((16 * s & (P - 1)) >> 4) * sub_size;
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
    tok = next_tok, next_tok = after_tok, source = next_source, page = next_page;
  }
}

template <int C>
int launch(const EvictArgs& a, int units, void* stream) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)units * C);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 2 : 1;
  return (int)cudaLaunchKernelEx(&cfg, akv_paged_evict_kernel<C>, a);
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
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return (int)e;
  // as many CTAs of a unit as are resident together, two an SM.  Microseconds with clusters of 1, 2, 4, 8: 256 units of 1.1 k tokens 26, 49, 81, 171; 16
  // of up to 32 k tokens 70, 50, 41, 27; 32 of 128 k tokens 675, 472, 264, 182.
  const int units = n * v.H, fit = 2 * sms / units;
  return fit >= 8 ? launch<8>(a, units, stream) : fit >= 4 ? launch<4>(a, units, stream) : fit >= 2 ? launch<2>(a, units, stream) : launch<1>(a, units, stream);
}

}  // namespace akv
