// Cuts sequences of a cache to a budget: of each key head's tokens the first, the last and those of the largest weights, copied in order to
// other blocks.
//
// Two kernels.  The first ranks: a cluster of CTAs has a (sequence, key head), each a part of its places.  Weights become 32-bit numbers that
// order like them (NaN lowest; what is kept in any case highest), which stay in shared memory; a radix selection of 11 + 11 + 10 bits finds the
// last number that is kept and how many of its equals are, each pass with one exchange of the counts over the cluster; then every warp
// knows how many kept places lie before its own and writes them to a list.  No order of atomics shows in it.
// The second copies: 64 places of the list (a group, which shares a scale in an 8-bit pool) are a warp's, rows in pieces of 16 bytes.
//
// What bounds them: latency the first (a launch, two dependent loads, three passes with an exchange each: 19 us for 32 sequences of 1900 to 2500
// places, 30 for one of 131072, 8 heads), the rows' bytes the second, which are read where the kept tokens happen to lie.  The former cut to 2048
// tokens, 128 dimensions, 4 bits: 55 us in all, 25 of bytes; the latter to a quarter, bf16: 87 us, 43 of bytes.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "kv.cuh"
#include "tc_ptx.cuh"

namespace spf {
namespace {

namespace cg = cooperative_groups;

constexpr int kMostParts = 8, kBins = 2048;
constexpr int kHeld = 36864;              // numbers that a CTA of the first kernel keeps (with more, they are made anew in every pass)
constexpr int kMoveThreads = 128;
constexpr uint32_t kAlways = 0xffffffffu;
constexpr int64_t kMostPlaces = 1 << 30;  // of a sequence, so that a place and what is added to it stay in 32 bits

struct EvictArgs {
  KvView kv;
  const int32_t *lens, *table, *keep, *to_table, *n_seen;
  int32_t* to_lens;
  int n_seqs, table_stride, to_stride, n_first, n_recent;
  float* weight;
  int32_t* position;
  int32_t* list;                          // [n_seqs][n_kv_heads][to_stride * block_tokens]: kept places
  int32_t* counts;                        // [n_seqs][n_kv_heads]
  int32_t* dev_status;
  int held;                               // numbers that fit into the first kernel's shared memory
};

__device__ __forceinline__ int64_t block_at(const KvView& kv, const int32_t* table, int stride, int seq, int pos) {
  const int b = __ldg(table + (int64_t)seq * stride + pos / kv.block_tokens);
  return b >= 0 && b < kv.n_blocks ? b : -1;
}
// Row of a place in the pools and the ledger, -1 outside.
__device__ __forceinline__ int64_t row_at(const KvView& kv, const int32_t* table, int stride, int seq, int head, int pos) {
  const int64_t b = block_at(kv, table, stride, seq, pos);
  return b < 0 ? -1 : (b * kv.n_kv_heads + head) * kv.block_tokens + pos % kv.block_tokens;
}

// A token's rank as a number.
__device__ __forceinline__ uint32_t rank_of(const EvictArgs& a, float w, int position, int64_t recent) {
  if (position < a.n_first || position >= recent) return kAlways;
  if (w != w) return 0u;
  const uint32_t bits = __float_as_uint(w + 0.f);        // -0 becomes 0
  return bits ^ ((bits >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}
// The ranks of four tokens from place pos on, a multiple of 4 (blocks are multiples of 128).
__device__ __forceinline__ uint4 ranks_at(const EvictArgs& a, int seq, int head, int pos, int64_t recent) {
  const int64_t row = row_at(a.kv, a.table, a.table_stride, seq, head, pos);
  float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
  int4 at = make_int4(0, 0, 0, 0);
  if (row >= 0) {
    w = __ldg(reinterpret_cast<const float4*>(a.weight + row));
    at = a.position != nullptr ? __ldg(reinterpret_cast<const int4*>(a.position + row)) : make_int4(pos, pos + 1, pos + 2, pos + 3);
  } else {
    report_cache(a.dev_status);
  }
  return make_uint4(rank_of(a, w.x, at.x, recent), rank_of(a, w.y, at.y, recent), rank_of(a, w.z, at.z, recent), rank_of(a, w.w, at.w, recent));
}

template <int kRankThreads>
struct RankSmem {
  static constexpr int kRankWarps = kRankThreads / 32;
  alignas(16) uint32_t bins[3][kBins];
  uint32_t sums[kRankWarps];
  uint32_t found[2];                      // bin, and what is left to be taken in it
  uint32_t above[kRankWarps + 1], equal[kRankWarps + 1];   // kept for certain, and candidates, before each warp; the last: of the CTA
};

template <int kRankThreads>
__global__ void __launch_bounds__(kRankThreads) rank_kernel(const __grid_constant__ EvictArgs a) {
  constexpr int kRankWarps = kRankThreads / 32;
  extern __shared__ __align__(16) uint32_t held[];
  __shared__ RankSmem<kRankThreads> sm;
  cg::cluster_group cluster = cg::this_cluster();
  const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int pair = (int)(blockIdx.x / parts), seq = pair / a.kv.n_kv_heads, head = pair - seq * a.kv.n_kv_heads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t room = (int64_t)a.to_stride * a.kv.block_tokens;
  int n = __ldg(a.lens + seq);
  if (n < 0 || n > (int64_t)a.table_stride * a.kv.block_tokens) {
    if (threadIdx.x == 0) report_cache(a.dev_status);
    n = 0;
  }
  const int left = (int)min((int64_t)min(n, max(__ldg(a.keep + seq), 0)), room);
  int32_t* list = a.list + (int64_t)pair * room;
  if (part == 0 && threadIdx.x == 0) a.counts[pair] = left;
  grid_launch_dependents();
  if (left == 0) return;
  // the CTA's places: chunks of 128, four to a lane
  const int each = ((n + parts - 1) / parts + 127) & ~127, lo = min(part * each, n), hi = min(lo + each, n);
  if (left == n) {
    for (int i = lo + (int)threadIdx.x; i < hi; i += kRankThreads) list[i] = i;
    return;
  }
  const int64_t recent = (int64_t)(a.n_seen != nullptr ? __ldg(a.n_seen + seq) : n) - a.n_recent;
  const bool fits = each <= a.held;
  uint4* held4 = reinterpret_cast<uint4*>(held);
  auto ranks = [&](int i) { return fits ? held4[(i - lo) / 4] : ranks_at(a, seq, head, i, recent); };
  for (int i = threadIdx.x; i < 3 * kBins; i += kRankThreads) (&sm.bins[0][0])[i] = 0;
  __syncthreads();
  uint32_t prefix = 0, take = (uint32_t)left;             // the last kept number's upper bits; kept ones among those that have them
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    auto count = [&](int i, const uint4& four) {
      const uint32_t r[4] = {four.x, four.y, four.z, four.w};
      uint32_t bin[4];
      bool counts[4], all = true;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        counts[j] = i + j < hi && (pass == 0 || (r[j] >> (shift + bits)) == prefix);
        bin[j] = (r[j] >> shift) & ((1u << bits) - 1u);
        all = all && counts[j] && bin[j] == bin[0];
      }
      // equal weights would be as many additions to one counter
      const uint32_t first = __shfl_sync(0xffffffffu, bin[0], 0);        // of every lane, not in a condition that some skip
      if (__all_sync(0xffffffffu, all && bin[0] == first)) {
        if (lane == 0) atomicAdd(&sm.bins[pass][bin[0]], 128u);
      } else if (all) {
        atomicAdd(&sm.bins[pass][bin[0]], 4u);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (counts[j]) atomicAdd(&sm.bins[pass][bin[j]], 1u);
      }
    };
    if (pass == 0) {
      // loads of four chunks in flight
      constexpr int kAhead = 4;
      for (int i0 = lo + warp * 128; i0 < hi; i0 += kAhead * kRankThreads * 4) {
        uint4 four[kAhead];
#pragma unroll
        for (int c = 0; c < kAhead; ++c) {
          const int i = i0 + c * kRankThreads * 4 + 4 * lane;
          four[c] = i < hi ? ranks_at(a, seq, head, i, recent) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int c = 0; c < kAhead; ++c) {
          const int i = i0 + c * kRankThreads * 4 + 4 * lane;
          if (i - 4 * lane >= hi) break;
          if (fits && i < hi) held4[(i - lo) / 4] = four[c];
          count(i, four[c]);
        }
      }
    } else {
      for (int i0 = lo + warp * 128; i0 < hi; i0 += kRankThreads * 4) {
        const int i = i0 + 4 * lane;
        count(i, i < hi ? ranks(i) : make_uint4(0u, 0u, 0u, 0u));
      }
    }
    cluster.sync();
    // every CTA adds up everybody's counts and finds the bin, from the highest number down
    constexpr int kPer = kBins / kRankThreads, kPairs = kPer / 2;
    uint32_t own[kPer] = {}, sum = 0;
#pragma unroll
    for (int pair = 0; pair < kPairs; ++pair) {
      const int at = kBins / 2 - 1 - ((int)threadIdx.x * kPairs + pair);
      uint2 counts[kMostParts];
#pragma unroll
      for (int p = 0; p < kMostParts; ++p)                // loads from all of them in flight together
        counts[p] = p < parts ? reinterpret_cast<const uint2*>(cluster.map_shared_rank(&sm.bins[pass][0], p))[at] : make_uint2(0u, 0u);
#pragma unroll
      for (int p = 0; p < kMostParts; ++p) own[2 * pair] += counts[p].y, own[2 * pair + 1] += counts[p].x;
      sum += own[2 * pair] + own[2 * pair + 1];
    }
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) sm.sums[warp] = upto;
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += sm.sums[w];
    uint32_t before = upto - sum;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (before < take && take <= before + own[j]) {
        sm.found[0] = (uint32_t)(kBins - 1 - (int)(threadIdx.x * kPer + j));
        sm.found[1] = take - before;
      }
      before += own[j];
    }
    __syncthreads();
    prefix = prefix << bits | sm.found[0];
    take = sm.found[1];
  }
  // kept: every number above `prefix`, and the first `take` that equal it
  __syncthreads();                                        // all numbers are held
  const int run = ((each / 128 + kRankWarps - 1) / kRankWarps) * 128, from = min(lo + warp * run, hi), to = min(from + run, hi);
  // of a lane's four: those above the number in the lower half, its equals in the upper one
  auto tally = [&](int i, const uint4& four) {
    uint32_t t = 0;
    const uint32_t r[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) t += i + j >= to ? 0u : r[j] > prefix ? 1u : r[j] == prefix ? 0x10000u : 0u;
    return t;
  };
  uint32_t above = 0, equal = 0;
  for (int i0 = from; i0 < to; i0 += 128) {
    const int i = i0 + 4 * lane;
    const uint32_t t = i < to ? tally(i, ranks(i)) : 0u;
    above += t & 0xffffu, equal += t >> 16;
  }
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) sm.above[warp] = above, sm.equal[warp] = equal;
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t u = 0, e = 0;
    for (int w = 0; w < kRankWarps; ++w) {
      const uint32_t du = sm.above[w], de = sm.equal[w];
      sm.above[w] = u, sm.equal[w] = e;
      u += du, e += de;
    }
    sm.above[kRankWarps] = u, sm.equal[kRankWarps] = e;
  }
  cluster.sync();
  above = sm.above[warp], equal = sm.equal[warp];
  for (int p = 0; p < part; ++p) {
    const RankSmem<kRankThreads>* other = cluster.map_shared_rank(&sm, p);
    above += other->above[kRankWarps], equal += other->equal[kRankWarps];
  }
  cluster.sync();                                         // nobody leaves while its counts are read
  for (int i0 = from; i0 < to; i0 += 128) {
    const int i = i0 + 4 * lane;
    const uint4 four = i < to ? ranks(i) : make_uint4(0u, 0u, 0u, 0u);
    const uint32_t t = i < to ? tally(i, four) : 0u;
    uint32_t upto = t;                                    // over the lanes up to this one: at most 128 of either
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    uint32_t u = above + ((upto - t) & 0xffffu), e = equal + ((upto - t) >> 16);
    const uint32_t r[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool more = i + j < to && r[j] > prefix, same = i + j < to && r[j] == prefix;
      if (more || (same && e < take)) list[u + min(e, take)] = i + j;
      u += more ? 1u : 0u;
      e += same ? 1u : 0u;
    }
    const uint32_t all = __shfl_sync(0xffffffffu, upto, 31);
    above += all & 0xffffu, equal += all >> 16;
  }
}

// Four E4M3 bytes times a ratio, rounded to nearest, clipped at 448 (NaN: 0x7F).
__device__ __forceinline__ uint32_t scale_bytes(uint32_t four, float ratio) {
  uint32_t lo, hi, r;
  asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(four));
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo)), y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  asm("{\n.reg .b16 a, b;\ncvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\nmov.b32 %0, {a, b};\n}"
      : "=r"(r)
      : "f"(x.x * ratio), "f"(x.y * ratio), "f"(y.x * ratio), "f"(y.y * ratio));
  return r;
}

template <int D, int BITS>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const __grid_constant__ EvictArgs a) {
  constexpr int kRow = D * BITS / 8, kPieces = kRow / 16, kLoads = 8, kWarps = kMoveThreads / 32;
  constexpr int kShares = kRow > 64 ? kRow / 64 : 1, kTokens = kScaleTokens / kShares;   // long rows: warps that share a group
  const int lane = threadIdx.x & 31;
  grid_wait();
  const int room_groups = a.to_stride * (a.kv.block_tokens / kScaleTokens);
  const int64_t room = (int64_t)room_groups * kScaleTokens, items = (int64_t)a.n_seqs * a.kv.n_kv_heads * room_groups * kShares;
  // warps on their own: an item is a chain of dependent loads (counts, table, list, table, rows), so the more are under way the better
  for (int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); item < items; item += (int64_t)gridDim.x * kWarps) {
    const int share = (int)(item % kShares);
    const int64_t whole = item / kShares;
    const int pair = (int)(whole / room_groups), group = (int)(whole - (int64_t)pair * room_groups);
    const int seq = pair / a.kv.n_kv_heads, head = pair - seq * a.kv.n_kv_heads, count = __ldg(a.counts + pair);
    if (group == 0 && head == 0 && share == 0 && lane == 0) a.to_lens[seq] = count;
    const int live = min(count - group * kScaleTokens, kScaleTokens), token0 = share * kTokens, token1 = min(token0 + kTokens, live);
    if (token0 >= token1) continue;
    const int64_t to = row_at(a.kv, a.to_table, a.to_stride, seq, head, group * kScaleTokens);
    if (to < 0) {
      if (lane == 0) report_cache(a.dev_status);
      continue;
    }
    int from[2];                                          // the rows in the pools of tokens lane and lane + 32, below zero: left out
    float scale[2][2], top[2];                            // 8 bits: of keys and values; the group's
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int token = lane + 32 * h;
      from[h] = -1;
      if (BITS == 8 ? token < live : token >= token0 && token < token1) {
        const int pos = __ldg(a.list + (int64_t)pair * room + group * kScaleTokens + token);
        from[h] = (int)row_at(a.kv, a.table, a.table_stride, seq, head, pos);
        if (from[h] < 0) report_cache(a.dev_status);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (from[h] >= 0 && lane + 32 * h >= token0 && lane + 32 * h < token1) {
        const int64_t cell = to + lane + 32 * h;
        const float weight = __ldg(a.weight + from[h]);
        const int position = a.position != nullptr ? __ldg(a.position + from[h]) : 0;
        a.weight[cell] = weight;
        if (a.position != nullptr) a.position[cell] = position;
      }
      if constexpr (BITS == 8) {
#pragma unroll
        for (int v = 0; v < 2; ++v) scale[v][h] = from[h] >= 0 ? __ldg((v ? a.kv.v_scale : a.kv.k_scale) + from[h] / kScaleTokens) : 0.f;
      }
    }
    if constexpr (BITS == 8) {
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        top[v] = fmaxf(scale[v][0], scale[v][1]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top[v] = fmaxf(top[v], __shfl_xor_sync(0xffffffffu, top[v], o));
        if (lane == 0 && share == 0 && top[v] > 0.f) (v ? a.kv.v_scale : a.kv.k_scale)[to / kScaleTokens] = top[v];
#pragma unroll
        for (int h = 0; h < 2; ++h) scale[v][h] = __fdiv_rn(scale[v][h], top[v]);      // what the tokens' bytes are multiplied by
      }
    }
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      uint8_t* pool = v ? a.kv.v : a.kv.k;
#pragma unroll 1
      for (int i0 = token0 * kPieces; i0 < token1 * kPieces; i0 += kLoads * 32) {
        uint4 x[kLoads];
        bool there[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int i = i0 + j * 32 + lane, token = i / kPieces;
          // kPieces divides 32 or is divided by it: the lanes' tokens of one j lie in one half
          const int first = i0 + j * 32 < kPieces * 32 ? from[0] : from[1];
          const int row = __shfl_sync(0xffffffffu, first, token & 31);
          float ratio = 1.f;
          if constexpr (BITS == 8) ratio = __shfl_sync(0xffffffffu, i0 + j * 32 < kPieces * 32 ? scale[v][0] : scale[v][1], token & 31);
          there[j] = i < token1 * kPieces && row >= 0;
          if (there[j]) {
            x[j] = __ldg(reinterpret_cast<const uint4*>(pool + (int64_t)row * kRow) + i % kPieces);
            if constexpr (BITS == 8) {
              if (ratio != 1.f) {
                x[j].x = scale_bytes(x[j].x, ratio), x[j].y = scale_bytes(x[j].y, ratio);
                x[j].z = scale_bytes(x[j].z, ratio), x[j].w = scale_bytes(x[j].w, ratio);
              }
            }
          }
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
          if (there[j]) reinterpret_cast<uint4*>(pool + to * kRow)[i0 + j * 32 + lane] = x[j];
      }
      if constexpr (BITS == 4) {
        constexpr int kWords = D / kScaleDims / 2;        // of a token's scales
        uint32_t* scales = reinterpret_cast<uint32_t*>(v ? a.kv.v_scale4 : a.kv.k_scale4);
        uint32_t x[2 * kWords];
#pragma unroll
        for (int j = 0; j < 2 * kWords; ++j) {
          const int i = j * 32 + lane, row = __shfl_sync(0xffffffffu, j < kWords ? from[0] : from[1], (i / kWords) & 31);
          x[j] = row >= 0 ? __ldg(scales + (int64_t)row * kWords + i % kWords) : 0u;
          if (row >= 0) scales[to * kWords + i] = x[j];
        }
      }
    }
  }
}

size_t list_bytes(const KvView& kv, int64_t n_seqs, int64_t to_stride) {
  return align_up((size_t)(n_seqs * kv.n_kv_heads) * (size_t)(to_stride * kv.block_tokens) * sizeof(int32_t), 256);
}
size_t evict_workspace(const KvView& kv, int64_t n_seqs, int64_t to_stride) {
  return list_bytes(kv, n_seqs, to_stride) + align_up((size_t)(n_seqs * kv.n_kv_heads) * sizeof(int32_t), 256);
}

int32_t check_cut(const char* who, const KvView& kv, int64_t n_seqs, int64_t to_stride) {
  if (n_seqs < 1 || n_seqs > (1 << 20) || to_stride < 1) return fail(SPF_ERR_INVALID_ARG, "%s: n_seqs and to_stride must be positive (n_seqs at most 2^20)", who);
  if (n_seqs * kv.n_kv_heads > (1 << 20)) return fail(SPF_ERR_UNSUPPORTED, "%s: more than 2^20 sequences times heads", who);
  if (to_stride * kv.block_tokens > kMostPlaces) return fail(SPF_ERR_UNSUPPORTED, "%s: to_stride * block_tokens is more than 2^30", who);
  return SPF_OK;
}

template <int D, int BITS>
int32_t launch_evict(EvictArgs& a, cudaStream_t stream) {
  // CTAs of a (sequence, key head): by the places that its table has room for, which is what the host knows.  One and four for 3000 places (the whole
  // call, 4 bits): 19 us either for a sequence, but 54 and 134 for 32 of them; two and eight for 8000 places: 19 and 23 us, 148 and 390.  A table wider
  // than its sequences costs as much: 2500 places in room for 131072, 22 us for a sequence, 226 for 32.
  const int64_t places = (int64_t)a.table_stride * a.kv.block_tokens, pairs = (int64_t)a.n_seqs * a.kv.n_kv_heads;
  const int parts = places <= 4096 ? 1 : places <= 8192 ? 2 : places <= 32768 ? 4 : kMostParts;
  a.held = (int)std::min<int64_t>(align_up((size_t)ceil_div(places, parts), 128), kHeld);
  // Few places: small CTAs, so that many sequences' run at the same time (32 sequences of 3000 tokens, 8 heads, the whole call: 256 threads 54 us, 1024 threads 60)
  static ContextSet done;
  const auto rank = parts == 1 ? rank_kernel<256> : rank_kernel<1024>;
  if (parts > 1) {
    const int32_t st = allow_shared_memory(reinterpret_cast<const void*>(rank_kernel<1024>), kHeld * 4, done);
    if (st != SPF_OK) return st;
  }
  cudaLaunchConfig_t config{};
  cudaLaunchAttribute attr{};
  config.gridDim = dim3((unsigned)(pairs * parts));
  config.blockDim = dim3(parts == 1 ? 256 : 1024);
  config.dynamicSmemBytes = (size_t)a.held * 4;
  config.stream = stream;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)parts;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  config.attrs = &attr;
  config.numAttrs = 1;
  SPF_CUDA_CHECK(cudaLaunchKernelEx(&config, rank, a));
  int sm_count = 0;
  if (const int32_t bad = device_sm_count(&sm_count); bad != SPF_OK) return bad;
  const int64_t items = pairs * a.to_stride * (a.kv.block_tokens / kScaleTokens) * std::max(D * BITS / 8 / 64, 1);
  config.gridDim = dim3((unsigned)std::min<int64_t>(ceil_div(items, kMoveThreads / 32), (int64_t)sm_count * 8));
  config.blockDim = dim3(kMoveThreads);
  config.dynamicSmemBytes = 0;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  SPF_CUDA_CHECK(cudaLaunchKernelEx(&config, move_kernel<D, BITS>, a));
  return SPF_OK;
}

}  // namespace

int32_t check_ledger(const char* who, const spf_kv_ledger* ledger) {
  if (ledger == nullptr || ledger->weight == nullptr) return fail(SPF_ERR_INVALID_ARG, "%s: ledger or its weight is null", who);
  if (reinterpret_cast<uintptr_t>(ledger->weight) % 16 != 0 || reinterpret_cast<uintptr_t>(ledger->position) % 16 != 0)
    return fail(SPF_ERR_INVALID_ARG, "%s: the ledger is not 16-byte aligned", who);
  return SPF_OK;
}

}  // namespace spf

using namespace spf;

extern "C" size_t spf_kv_evict_workspace_bytes(const spf_kv_cache* cache, int32_t n_seqs, int32_t to_stride) {
  const char* who = "spf_kv_evict_workspace_bytes";
  clear_error();
  KvView kv;
  if (check_cache(who, cache, &kv) != SPF_OK || check_cut(who, kv, n_seqs, to_stride) != SPF_OK) return 0;
  return evict_workspace(kv, n_seqs, to_stride);
}

extern "C" int32_t spf_kv_evict(const spf_kv_cache* cache, const spf_kv_ledger* ledger, const spf_kv_cut* cut, void* workspace, size_t workspace_bytes,
                                int32_t* dev_status, void* cuda_stream) {
  const char* who = "spf_kv_evict";
  clear_error();
  EvictArgs a{};
  int32_t st = check_cache(who, cache, &a.kv);
  if (st == SPF_OK) st = check_ledger(who, ledger);
  if (st != SPF_OK) return st;
  if (cut == nullptr) return fail(SPF_ERR_INVALID_ARG, "%s: cut is null", who);
  st = check_cut(who, a.kv, cut->n_seqs, cut->to_stride);
  if (st != SPF_OK) return st;
  if (cut->table_stride < 1) return fail(SPF_ERR_INVALID_ARG, "%s: table_stride must be positive", who);
  if ((int64_t)cut->table_stride * a.kv.block_tokens > kMostPlaces) return fail(SPF_ERR_UNSUPPORTED, "%s: table_stride * block_tokens is more than 2^30", who);
  if (cut->n_first < 0 || cut->n_recent < 0) return fail(SPF_ERR_INVALID_ARG, "%s: n_first and n_recent must not be negative", who);
  if (cut->seq_lens == nullptr || cut->block_table == nullptr || cut->keep == nullptr || cut->to_table == nullptr || cut->to_lens == nullptr)
    return fail(SPF_ERR_INVALID_ARG, "%s: seq_lens, block_table, keep, to_table or to_lens is null", who);
  const size_t need = evict_workspace(a.kv, cut->n_seqs, cut->to_stride);
  if (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return fail(SPF_ERR_WORKSPACE, "%s: workspace is null or not 256-byte aligned", who);
  if (workspace_bytes < need) return fail(SPF_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, need);
  a.lens = cut->seq_lens, a.table = cut->block_table, a.keep = cut->keep, a.to_table = cut->to_table, a.n_seen = cut->n_seen;
  a.to_lens = cut->to_lens;
  a.n_seqs = cut->n_seqs, a.table_stride = cut->table_stride, a.to_stride = cut->to_stride, a.n_first = cut->n_first, a.n_recent = cut->n_recent;
  a.weight = ledger->weight, a.position = ledger->position;
  a.list = static_cast<int32_t*>(workspace);
  a.counts = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + list_bytes(a.kv, cut->n_seqs, cut->to_stride));
  a.dev_status = dev_status;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool d64 = cache->head_dim == 64;
  switch (a.kv.bits) {
    case 4: return d64 ? launch_evict<64, 4>(a, stream) : launch_evict<128, 4>(a, stream);
    case 8: return d64 ? launch_evict<64, 8>(a, stream) : launch_evict<128, 8>(a, stream);
    default: return d64 ? launch_evict<64, 16>(a, stream) : launch_evict<128, 16>(a, stream);
  }
}
