// Attention of a step with many rows per key head (chunks of prompts) over the paged cache, bf16, 8 or 4 bits: the formulas, masks and
// references of the kernel for few rows, with the products on the big tensor-core instruction.
//
// A CTA works on 256 rows of a (sequence, key head), two tiles X of 128, against tiles of 128 keys.  Per tile of keys
//   S_X = Q_X K^T            128 x 128, into tensor memory,
//   P_X = 2^(c S_X - m)      by 128 threads, one to a row, back into the columns of S_X, rounded to bf16 (8-bit caches: fp16),
//   O_X += P_X V             P_X from tensor memory, V from shared memory as it lies there (dimensions contiguous).
// While the products of one row tile run, the threads of the other take their exponentials, so the two units that bound it, the
// tensor cores and the exponential unit (128 x 128 of either take about as long for 128 dimensions), overlap.  S_X for the
// next keys is asked for when O_X's product is done, which reads P_X from the same columns.
//
// The work is dealt out as for few rows: the list of all key tiles of all (sequence, row tile, key head) triples, up to a row tile's
// last visible key, is cut into one part for each SM; parts of a triple meet in a second kernel.
//
// Two row tiles and 128 keys take about 3400 cycles at 128 dimensions, of which the tensor cores are busy 2048 and the exponential unit
// 2048 (2048 new of 32k tokens, calls back to back: 505 us, 1055 TFLOP/s, at the clock that the power limit leaves).  Not taken, all slower there: a part
// of the exponentials as polynomials on the multiply-add units, products with the first half of the weights while the second is made,
// logits read in two halves, exponentials of the two row tiles strictly in turns.
//
// Warps: 0-3 and 4-7 the rows of the two tiles (softmax, rescaling of O where a reference moves, output), 8-11 queries and values
// (below), 12 copies, 13 issues the products.
//
// Queries: read once per triple by warps 8-11; 8 bits: as an E4M3 and an E5M2 term, as for few rows, so that 8-bit keys are
// multiplied as they are.  Values of 8-bit caches are widened to fp16 by these warps between their copy and their product; keys and values of
// 4-bit caches to bf16, which holds scale times (code - 8) exactly, so that everything else is as over a bf16 cache.
// Values of bf16 caches go straight from the copy to the product, but for tiles at the ends of a sequence's range, where
// what lies outside is cleared (a weight of zero would make NaN of NaN), and tiles whose last keys only later rows may see: values
// there that are not finite are cleared and put down with their place, and the output's rows that do see them get them back.
#include <algorithm>

#include "attend.cuh"

namespace spf {
namespace {

constexpr int kRows = 256, kKeys = 128, kThreads = 512;
constexpr int kSoftmaxRegs = 184, kOtherRegs = 72;    // of 128 a thread at launch: 256 x (184 + 72) = 512 x 128
constexpr int kInfo = 8;                              // tiles' scales kept: more than may be under way between copy and softmax
constexpr int kNever = 0x7fffffff;

template <int D_, int BITS_>
struct Traits {
  static constexpr int D = D_;
  static constexpr bool FP8 = BITS_ == 8, INT4 = BITS_ == 4;
  static constexpr int ROWB = FP8 ? D : 2 * D, SPAN = ROWB < 128 ? ROWB : 128;   // bytes of a row of keys in the products, and of the swizzle's span
  static constexpr int QTILE = 128 * D * 2;                                     // bf16, or two 8-bit terms
  static constexpr int KTILE = kKeys * ROWB, V8TILE = FP8 ? kKeys * D : 0, VTILE = kKeys * D * 2;
  static constexpr int STAGES = D == 64 ? 3 : 2;
  // 4 bits: a copied tile of keys or of values, the scales behind the codes, and how many of either are under way (one where there is no room
  // for more: it is widened in a tenth of the time that the products of a tile take, which is left for the next copy)
  static constexpr int PARTS = D / kScaleDims, CODES = kKeys * D / 2, RAW = INT4 ? CODES + kKeys * PARTS * 2 : 0, RAWS = D == 64 ? 3 : 1;
  static constexpr int QBUFS = D == 64 ? 2 : 1;                                 // where there is room, the next part's queries are fetched ahead
  // Tensor memory, 512 columns: S_X 128 each, O_X D each.  With 64 dimensions there is room for P_X (64 each) beside S_X, and the
  // next keys' logits are made while these are being turned into weights; with 128, P_X lies over S_X.
  static constexpr bool APART = D == 64;
  static constexpr uint32_t O_COL = 256, P_COL = APART ? 384 : 0, P_STEP = APART ? 64 : 128;
  static constexpr int BYTES = QBUFS * 2 * QTILE + STAGES * (KTILE + V8TILE + VTILE) + RAWS * 2 * RAW;
};

// What the copying warp tells the others about a part of a triple.
struct Part {
  int row0, n_new, pos0, first, end, head, row_tile, tile0, n_tiles, live, flags, behind;
  int dirty;                           // some value was put down in `bad`
  int bad[3][128];                     // per dimension, the first key that has NaN, +inf, -inf there (of those that were cleared)
  float q_factor[kRows];               // 8 bits
};
enum : int { kFromStart = 1, kToEnd = 2 };

struct TileInfo {
  float k_scale[2], v_log2[2];         // of the tile's two groups of 64 keys
};

struct Smem {
  unsigned long long s_full[2], s_free[2], p_ready[2], o_done[2], o_free[2], q_ready[2], q_free[2], part_full[2], part_empty[2], values_done[2], mma_done;
  unsigned long long k_full[3], k_empty[3], v_full[3], v_ready[3], v_empty[3], v8_empty[3], k4_full[3], k4_empty[3];
  TileInfo info[kInfo];
  Part part[2];
  int64_t scan[kThreads / 32];
  int64_t total, start_base;
  int start_seq, start_tile;
  int abort;
  uint32_t tmem;
};

template <class T>
constexpr int smem_bytes() { return T::BYTES + (int)sizeof(Smem) + 1024; }

struct PromptArgs {
  AttendArgs a;
  CUtensorMap k_map, v_map;
  CUtensorMap k_scale_map, v_scale_map;                // 4 bits
  AttendParts parts;
};

// ---------------------------------------------------------------------------------------------- the list of tiles
__device__ __forceinline__ int row_tiles_of(const AttendArgs& a, const SeqSpan& s) { return (int)(((int64_t)s.n_new * a.group + kRows - 1) / kRows); }
// Key behind the last one that any row of a row tile may see.
__device__ __forceinline__ int keys_end(const AttendArgs& a, const SeqSpan& s, int row_tile) {
  if (!a.causal) return s.end;
  const int last = (int)min(((int64_t)(row_tile + 1) * kRows - 1) / a.group, (int64_t)s.n_new - 1);
  return max(min(s.end, s.pos0 + last + 1), s.first);
}
// Tiles of a triple in the list: at least one, also for rows without keys, whose output is zeros.
__device__ __forceinline__ int tiles_of(const AttendArgs& a, const SeqSpan& s, int row_tile) {
  return max((keys_end(a, s, row_tile) + kKeys - 1) / kKeys - s.first / kKeys, 1);
}

// Length of the list, and the (sequence, row tile) that holds the CTA's first tile.
__device__ __forceinline__ void find_start(const PromptArgs& args, Smem& sm) {
  const AttendArgs& a = args.a;
  const int run = (a.step.n_seqs + kThreads - 1) / kThreads, lo = min((int)threadIdx.x * run, a.step.n_seqs), hi = min(lo + run, a.step.n_seqs);
  int64_t mine = 0;
  for (int b = lo; b < hi; ++b) {
    const SeqSpan s = seq_span(a, b);
    const int n = row_tiles_of(a, s);
    for (int t = 0; t < n; ++t) mine += (int64_t)a.kv.n_kv_heads * tiles_of(a, s, t);
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sm.scan[warp] = upto;
  __syncthreads();
  int64_t total = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) upto += sm.scan[w];
    total += sm.scan[w];
  }
  const int64_t w0 = (total + gridDim.x - 1) / gridDim.x * blockIdx.x;
  if (threadIdx.x == 0) sm.total = total;
  if (w0 >= upto - mine && w0 < upto) {
    int64_t base = upto - mine;
    for (int b = lo; b < hi; ++b) {
      const SeqSpan s = seq_span(a, b);
      const int n = row_tiles_of(a, s);
      bool found = false;
      for (int t = 0; t < n && !found; ++t) {
        const int64_t cost = (int64_t)a.kv.n_kv_heads * tiles_of(a, s, t);
        if (w0 < base + cost) {
          sm.start_seq = b;
          sm.start_tile = t;
          sm.start_base = base;
          found = true;
        } else {
          base += cost;
        }
      }
      if (found) break;
    }
  }
  __syncthreads();
}

// ---------------------------------------------------------------------------------------------- copies
template <class T>
__device__ __forceinline__ void copy_tiles(const PromptArgs& args, Smem& sm, uint32_t k_ring, uint32_t v_ring, int64_t w0, int64_t w1, int64_t per,
                                           const Abort& ab) {
  const AttendArgs& a = args.a;
  const int lane = threadIdx.x & 31;
  const int64_t pool_rows = a.kv.n_blocks * a.kv.n_kv_heads * a.kv.block_tokens;
  int seq = sm.start_seq, row_tile = sm.start_tile, n_parts = 0;
  int64_t base = sm.start_base, issued = 0;
  SeqSpan s = seq_span(a, seq);
  for (int64_t w = w0; w < w1;) {
    int tiles = tiles_of(a, s, row_tile);
    while (w >= base + (int64_t)a.kv.n_kv_heads * tiles) {
      base += (int64_t)a.kv.n_kv_heads * tiles;
      ++row_tile;
      while (row_tile >= row_tiles_of(a, s)) {           // sequences without rows are passed over
        s = seq_span(a, ++seq);
        row_tile = 0;
      }
      tiles = tiles_of(a, s, row_tile);
    }
    const int64_t in = w - base;
    const int head = (int)(in / tiles), skip = (int)(in - (int64_t)head * tiles);
    const int64_t to = base + (int64_t)(head + 1) * tiles;
    const bool empty = keys_end(a, s, row_tile) <= s.first;
    const int count = (int)(min(to, w1) - w);
    const int slot = n_parts & 1;
    if (n_parts >= 2 && !mbar_wait_warp(smem_u32(&sm.part_empty[slot]), (uint32_t)(n_parts / 2 - 1) & 1u, ab)) return;
    Part& part = sm.part[slot];
    for (int i = lane; i < 3 * 128; i += 32) part.bad[i >> 7][i & 127] = kNever;
    if (lane == 0) {
      part.row0 = s.row0, part.n_new = s.n_new, part.pos0 = s.pos0, part.first = s.first, part.end = s.end;
      part.head = head, part.row_tile = row_tile;
      part.tile0 = s.first / kKeys + skip;
      part.n_tiles = empty ? 0 : count;
      part.live = (int)min((int64_t)kRows, (int64_t)s.n_new * a.group - (int64_t)row_tile * kRows);
      part.flags = (skip == 0 ? kFromStart : 0) | (to <= w1 ? kToEnd : 0);
      part.behind = (int)((to - 1) / per - blockIdx.x);
      part.dirty = 0;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.part_full[slot]));
    ++n_parts;
    const int tile0 = s.first / kKeys + skip;
    for (int j0 = 0; !empty && j0 < count; j0 += 32) {
      // each lane looks one of the next 32 tiles up
      int row = 0;
      TileInfo info{};
      if (j0 + lane < count) {
        row = pool_row(a, seq, head, (tile0 + j0 + lane) * kKeys);
        if constexpr (T::FP8) {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const int key = (tile0 + j0 + lane) * kKeys + g * kScaleTokens, at = row + g * kScaleTokens;
            info.k_scale[g] = a.c * group_scale(a.kv.k_scale, s, key, at, pool_rows);
            info.v_log2[g] = log2f(group_scale(a.kv.v_scale, s, key, at, pool_rows));
          }
        }
      }
      for (int j = 0; j < min(32, count - j0); ++j, ++issued) {
        if constexpr (T::INT4) {
          const int raw = (int)(issued % T::RAWS);
          const uint32_t before = ((uint32_t)(issued / T::RAWS) & 1u) ^ 1u;
          if (!mbar_wait_warp(smem_u32(&sm.k4_empty[raw]), before, ab)) return;
          if (lane == j) {
            const uint32_t bar = smem_u32(&sm.k4_full[raw]), at = v_ring + 2 * raw * T::RAW;
            mbar_expect_tx(bar, T::RAW);
            tma_load_3d(at, &args.k_map, 0, row, 0, bar);
            tma_load_2d(at + T::CODES, &args.k_scale_map, 0, row / kKeys, bar);
          }
          if (!mbar_wait_warp(smem_u32(&sm.v8_empty[raw]), before, ab)) return;
          if (lane == j) {
            const uint32_t bar = smem_u32(&sm.v_full[raw]), at = v_ring + (2 * raw + 1) * T::RAW;
            mbar_expect_tx(bar, T::RAW);
            tma_load_3d(at, &args.v_map, 0, row, 0, bar);
            tma_load_2d(at + T::CODES, &args.v_scale_map, 0, row / kKeys, bar);
          }
          continue;
        }
        const int stage = (int)(issued % T::STAGES);
        const uint32_t parity = (uint32_t)(issued / T::STAGES) & 1u;
        if (!mbar_wait_warp(smem_u32(&sm.k_empty[stage]), parity ^ 1u, ab)) return;
        if (lane == j) {
          if constexpr (T::FP8) sm.info[issued % kInfo] = info;
          const uint32_t bar = smem_u32(&sm.k_full[stage]);
          mbar_expect_tx(bar, T::KTILE);
          tma_load_3d(k_ring + stage * T::KTILE, &args.k_map, 0, row, 0, bar);
        }
        if (!mbar_wait_warp(smem_u32(T::FP8 ? &sm.v8_empty[stage] : &sm.v_empty[stage]), parity ^ 1u, ab)) return;
        if (lane == j) {
          const uint32_t bar = smem_u32(&sm.v_full[stage]);
          mbar_expect_tx(bar, T::KTILE);
          tma_load_3d(v_ring + stage * T::KTILE, &args.v_map, 0, row, 0, bar);
        }
      }
    }
    w += count;
  }
  // no more parts
  const int slot = n_parts & 1;
  if (n_parts >= 2 && !mbar_wait_warp(smem_u32(&sm.part_empty[slot]), (uint32_t)(n_parts / 2 - 1) & 1u, ab)) return;
  if (lane == 0) {
    sm.part[slot].live = 0;
    mbar_arrive(smem_u32(&sm.part_full[slot]));
  }
}

// The next part, nullptr when there is none (or the CTA gives up).
struct PartReader {
  int n = 0;
  __device__ __forceinline__ Part* next(Smem& sm, const Abort& ab) {
    if (!mbar_wait_warp(smem_u32(&sm.part_full[n & 1]), (uint32_t)(n >> 1) & 1u, ab)) return nullptr;
    Part* p = &sm.part[n & 1];
    return p->live > 0 ? p : nullptr;
  }
  // One arrival a warp.
  __device__ __forceinline__ void done(Smem& sm) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&sm.part_empty[n & 1]));
    ++n;
  }
};

// ---------------------------------------------------------------------------------------------- queries and values
// Eight bf16 elements in the order in which codes come out of a word: 0 4 1 5 2 6 3 7.
__device__ __forceinline__ uint4 code_order(const uint4& v) {
  return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}
__device__ __forceinline__ constexpr int code_place(int i) { return (i & ~7) + ((i & 1) << 2) + ((i & 7) >> 1); }   // element in place i of that order

// Eight codes as bf16 elements, in that order.  A code shifted to the upper bits of 16.0's mantissa makes 16 + code, exactly, and so is its
// product with the scale less 24 scales (at most five significant bits in a scale, eight in either term's and the result's).
__device__ __forceinline__ uint4 widen_codes(uint32_t w, uint32_t scales, uint32_t less) {
  uint32_t r[4] = {w << 3, w >> 1, w >> 5, w >> 9};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = (r[i] & 0x00780078u) | 0x41804180u;
    asm("fma.rn.bf16x2 %0, %0, %1, %2;" : "+r"(r[i]) : "r"(scales), "r"(less));
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Widens a tile of codes, rows of 2 D bytes in spans of 128 as the products read them.  VALUES: keys outside [first, end) become zeros, and
// elements that are not finite (those of a scale that is not) of keys from `all` on are cleared and put down.
template <class T, bool VALUES>
__device__ __forceinline__ void widen_tile(Part& p, const unsigned char* raw, unsigned char* tile, int thread, int key0, int first, int end, int all) {
#pragma unroll 2
  for (int item = thread; item < kKeys * T::PARTS; item += 128) {
    const int k = item / T::PARTS, c = item % T::PARTS, key = key0 + k;
    const uint4 codes = *reinterpret_cast<const uint4*>(raw + (T::D == 128 ? k * 64 + ((c ^ (k >> 1)) & 3) * 16 : k * 32 + ((c ^ (k >> 2)) & 1) * 16));
    uint32_t scale = *reinterpret_cast<const uint16_t*>(raw + T::CODES + (k * T::PARTS + c) * 2);
    if (VALUES) {
      if (key < first || key >= end) {
        scale = 0;
      } else if (key >= all && (scale & 0x7f80u) == 0x7f80u) {
        for (int i = 0; i < kScaleDims; ++i) atomicMin(&p.bad[0][c * kScaleDims + i], key);
        p.dirty = 1;
        scale = 0;
      }
    }
    const uint32_t both = scale | scale << 16;
    uint32_t less;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(less) : "r"(both), "r"(0xc1c0c1c0u));      // -24
    unsigned char* dst = tile + (c >> 1) * (kKeys * 128) + k * 128;
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(dst + (((4 * c + i) ^ k) & 7) * 16) = widen_codes(w[i], both, less);
  }
}

template <class T>
__device__ __forceinline__ void load_queries(const AttendArgs& a, Part& p, unsigned char* q_tiles, int thread) {
  constexpr int D = T::D, kLanes = D / 8, kBatch = T::FP8 ? 2 : 8;    // loads in flight (8 bits: their conversions are long; 8: 600 instead of 550 us)
  static_assert(kRows * kLanes % (128 * kBatch) == 0);
  const uint32_t group = (uint32_t)a.group, first = (uint32_t)p.row_tile * kRows, total = (uint32_t)p.n_new * group;
  const int part = thread % kLanes;
  const __nv_bfloat16* heads = a.q.data + (int64_t)p.row0 * a.q.stride_row + (int64_t)p.head * a.group * a.q.stride_head + 8 * part;
#pragma unroll 1
  for (int r0 = thread / kLanes; r0 < kRows; r0 += kBatch * (128 / kLanes)) {
    union { uint4 u; __nv_bfloat162 h[4]; } v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const uint32_t rr = first + (uint32_t)(r0 + i * (128 / kLanes)), token = rr / group, g = rr - token * group;
      v[i].u = make_uint4(0, 0, 0, 0);
      if (rr < total) v[i].u = __ldg(reinterpret_cast<const uint4*>(heads + token * a.q.stride_row + g * a.q.stride_head));
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = r0 + i * (128 / kLanes), x = r >> 7, in = r & 127;
      unsigned char* tile = q_tiles + x * T::QTILE;
      if constexpr (!T::FP8) {
        if constexpr (T::INT4) v[i].u = code_order(v[i].u);
        *reinterpret_cast<uint4*>(tile + (part >> 3) * (128 * 128) + in * 128 + ((part ^ in) & 7) * 16) = v[i].u;
      } else {
        float f[8], top = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 t = __bfloat1622float2(v[i].h[j]);
          f[2 * j] = t.x, f[2 * j + 1] = t.y;
          top = fmaxf(top, fmaxf(fabsf(t.x), fabsf(t.y)));
        }
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o, kLanes));
        int e;
        uint2 hi, lo;
        two_terms(f, top, &e, &hi, &lo);
        const int chunk = part >> 1;
        unsigned char* at = tile + (D == 128 ? in * 128 + ((chunk ^ in) & 7) * 16 : in * 64 + ((chunk ^ (in >> 1)) & 3) * 16) + 8 * (part & 1);
        *reinterpret_cast<uint2*>(at) = hi;
        *reinterpret_cast<uint2*>(at + 128 * D) = lo;
        if (part == 0) p.q_factor[r] = __uint_as_float((uint32_t)(127 - e) << 23);
      }
    }
  }
}

// Clears what is not finite among 16 bytes of values (of a key, from dimension `dim` on) and puts it down.  Apart from the loop that
// looks for such bytes, so that what is hardly ever needed does not crowd its instructions out.
template <bool FP8>
__device__ __noinline__ uint4 put_down(Part& p, uint4 raw, int dim, int key) {
  uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll 1
    for (int i = 0; i < (FP8 ? 4 : 2); ++i) {
      const uint32_t bits = FP8 ? 0xffu << (8 * i) : 0xffffu << (16 * i), v = (w[j] & bits) >> (FP8 ? 8 * i : 16 * i);
      const bool nan = FP8 ? (v & 0x7fu) == 0x7fu : (v & 0x7fffu) > 0x7f80u, infinite = !FP8 && (v & 0x7fffu) == 0x7f80u;
      if (nan || infinite) {
        atomicMin(&p.bad[nan ? 0 : (v & 0x8000u) ? 2 : 1][dim + (FP8 ? 4 : 2) * j + i], key);
        p.dirty = 1;
        w[j] &= ~bits;
      }
    }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Whether any of 16 bytes of values is not finite: the exponent (E4M3: all but the sign) of ones overflows into the sign's place.
template <bool FP8>
__device__ __forceinline__ bool any_not_finite(const uint4& v) {
  constexpr uint32_t kBits = FP8 ? 0x7f7f7f7fu : 0x7f807f80u, kOne = FP8 ? 0x01010101u : 0x00800080u, kSign = FP8 ? 0x80808080u : 0x80008000u;
  return ((((v.x & kBits) + kOne) | ((v.y & kBits) + kOne) | ((v.z & kBits) + kOne) | ((v.w & kBits) + kOne)) & kSign) != 0;
}

template <class T>
__device__ __forceinline__ void prepare_values(const AttendArgs& a, Smem& sm, unsigned char* q_tiles, unsigned char* k_ring, unsigned char* v8_ring,
                                               unsigned char* v_ring, const Abort& ab) {
  constexpr int D = T::D;
  const int thread = threadIdx.x - 256, lane = threadIdx.x & 31;
  PartReader reader;
  int64_t used = 0;
  int with_keys = 0;
  while (Part* pp = reader.next(sm, ab)) {
    Part& p = *pp;
    if (p.n_tiles > 0) {
      const int buf = with_keys % T::QBUFS, round = with_keys / T::QBUFS;
      if (round > 0 && !mbar_wait_warp(smem_u32(&sm.q_free[buf]), (uint32_t)(round - 1) & 1u, ab)) return;
      ++with_keys;
      load_queries<T>(a, p, q_tiles + buf * 2 * T::QTILE, thread);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.q_ready[buf]));
    }
    const int seen_by_all = a.causal ? p.pos0 + (int)((int64_t)p.row_tile * kRows / a.group) + 1 : p.end;   // keys below this one
    for (int j = 0; j < p.n_tiles; ++j, ++used) {
      const int stage = (int)(used % T::STAGES);
      const uint32_t parity = (uint32_t)(used / T::STAGES) & 1u;
      if constexpr (T::INT4) {
        const int raw = (int)(used % T::RAWS), key0 = (p.tile0 + j) * kKeys;
        const uint32_t raw_parity = (uint32_t)(used / T::RAWS) & 1u;
        if (!mbar_wait_warp(smem_u32(&sm.k4_full[raw]), raw_parity, ab)) return;
        if (!mbar_wait_warp(smem_u32(&sm.k_empty[stage]), parity ^ 1u, ab)) return;
        widen_tile<T, false>(p, v8_ring + 2 * raw * T::RAW, k_ring + stage * T::KTILE, thread, key0, p.first, p.end, seen_by_all);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&sm.k_full[stage]));
          mbar_arrive(smem_u32(&sm.k4_empty[raw]));
        }
        if (!mbar_wait_warp(smem_u32(&sm.v_full[raw]), raw_parity, ab)) return;
        if (!mbar_wait_warp(smem_u32(&sm.v_empty[stage]), parity ^ 1u, ab)) return;
        widen_tile<T, true>(p, v8_ring + (2 * raw + 1) * T::RAW, v_ring + stage * T::VTILE, thread, key0, p.first, p.end, seen_by_all);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&sm.v_ready[stage]));
          mbar_arrive(smem_u32(&sm.v8_empty[raw]));
        }
        continue;
      }
      if (!mbar_wait_warp(smem_u32(&sm.v_full[stage]), parity, ab)) return;
      if constexpr (T::FP8) {
        if (!mbar_wait_warp(smem_u32(&sm.v_empty[stage]), parity ^ 1u, ab)) return;
      }
      const int key0 = (p.tile0 + j) * kKeys;
      const bool ends = key0 < p.first || key0 + kKeys > p.end, later = key0 + kKeys > seen_by_all;
      unsigned char* tile = v_ring + stage * T::VTILE;
      if constexpr (T::FP8) {
        const unsigned char* src = v8_ring + stage * T::V8TILE;
        // One piece at a time: the roles' instructions share a cache, and four at a time took 496 instead of 465 us (two: 478).
#pragma unroll 1
        for (int item = thread; item < kKeys * (D / 16); item += 128) {
          const int k = item / (D / 16), c = item % (D / 16), key = key0 + k;
          uint4 raw = *reinterpret_cast<const uint4*>(src + (D == 128 ? k * 128 + ((c ^ k) & 7) * 16 : k * 64 + ((c ^ (k >> 1)) & 3) * 16));
          if (ends && (key < p.first || key >= p.end)) raw = make_uint4(0, 0, 0, 0);
          if (later && key >= seen_by_all && any_not_finite<true>(raw)) raw = put_down<true>(p, raw, c * 16, key);
          uint32_t o[8];
          const uint32_t* w = &raw.x;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t even, odd;
            widen4(w[i], even, odd);
            o[2 * i] = __byte_perm(even, odd, 0x5410);
            o[2 * i + 1] = __byte_perm(even, odd, 0x7632);
          }
          unsigned char* dst = tile + (c >> 2) * (kKeys * 128) + k * 128;
          *reinterpret_cast<uint4*>(dst + (((2 * c) ^ k) & 7) * 16) = make_uint4(o[0], o[1], o[2], o[3]);
          *reinterpret_cast<uint4*>(dst + (((2 * c + 1) ^ k) & 7) * 16) = make_uint4(o[4], o[5], o[6], o[7]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      } else if (ends || later) {
        for (int item = thread; item < kKeys * (D / 8); item += 128) {
          const int k = item / (D / 8), c = item % (D / 8), key = key0 + k;
          uint4* at = reinterpret_cast<uint4*>(tile + (c >> 3) * (kKeys * 128) + k * 128 + ((c ^ k) & 7) * 16);
          if (key < p.first || key >= p.end) {
            *at = make_uint4(0, 0, 0, 0);
          } else if (key >= seen_by_all) {
            const uint4 raw = *at;
            if (any_not_finite<false>(raw)) *at = put_down<false>(p, raw, c * 8, key);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(smem_u32(&sm.v_ready[stage]));
        if constexpr (T::FP8) mbar_arrive(smem_u32(&sm.v8_empty[stage]));
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.values_done[reader.n & 1]));
    reader.done(sm);
  }
}

// ---------------------------------------------------------------------------------------------- products
// The issuing warp goes through its loop as a whole and one lane's predicate is on the instructions alone: operands then are values
// that the whole warp shares, which is where the instructions want them.  (One thread in a branch of its own had to bring each of an
// instruction's six operand registers there: 75 to 115 cycles an instruction that takes the tensor cores 64.)
//
// D[128 x N] (+)= A . B^T, both operands in shared memory: 16 bf16, or 32 bytes, of a row.
template <bool FP8>
__device__ __forceinline__ void mma_from_smem(uint32_t lane_on, uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
#define SPF_MMA(KIND)                                                                                                                  \
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::" KIND              \
               " [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(lane_on)                \
               : "memory")
  if constexpr (FP8) SPF_MMA("f8f6f4");
  else SPF_MMA("f16");
#undef SPF_MMA
}
// D[128 x N] (+)= A[128 x 16] . B: A from tensor memory, 16 bits.
__device__ __forceinline__ void mma_from_tmem(uint32_t lane_on, uint32_t d, uint32_t a, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
               "r"(a), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(lane_on)
               : "memory");
}
__device__ __forceinline__ void commit(uint32_t lane_on, uint32_t bar) {
  asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"(lane_on)
               : "memory");
}
// Operand whose columns (dimensions) are contiguous: blocks of 64 of them, kKeys rows of 128 bytes each (128-byte swizzle), one
// behind the other; 8 rows (keys) are 1024 bytes.
__device__ __forceinline__ uint64_t value_desc(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((kKeys * 128) >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

template <class T>
__device__ __forceinline__ void logits(uint32_t lane_on, uint32_t s, uint64_t q, uint64_t k) {
  constexpr uint32_t idesc = instr_desc(128, kKeys, T::FP8);
  if constexpr (T::FP8) {
    // the second term's format is E5M2
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int ks = 0; ks < T::SPAN / 32; ++ks)
        mma_from_smem<true>(lane_on, s, q + (uint32_t)(t * (128 * T::D >> 4) + 2 * ks), k + 2u * ks, t == 0 ? idesc : idesc | (1u << 7),
                            (uint32_t)((t | ks) != 0));
  } else {
#pragma unroll
    for (int i = 0; i < T::D / 16; ++i) {
      const uint32_t at = (uint32_t)((i >> 2) * (128 * 128 >> 4) + 2 * (i & 3));
      mma_from_smem<false>(lane_on, s, q + at, k + at, idesc, (uint32_t)(i != 0));
    }
  }
}
template <class T>
__device__ __forceinline__ void weigh(uint32_t lane_on, uint32_t o, uint32_t p, uint64_t v, uint32_t accumulate) {
  constexpr uint32_t type = T::FP8 ? 0u : 1u;            // fp16 or bf16; the right operand's columns are contiguous (bit 16)
  constexpr uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | (1u << 16) | ((uint32_t)(T::D >> 3) << 17) | (8u << 24);
#pragma unroll
  for (int ks = 0; ks < kKeys / 16; ++ks)
    mma_from_tmem(lane_on, o, p + 8 * ks, v + (uint32_t)(ks * (2048 >> 4)), idesc, ks == 0 ? accumulate : 1u);
}

// The order of the products.  Where weights lie over logits: per row tile, tile j's values, then tile j + 1's logits; the other row
// tile's threads are busy meanwhile.  Where they lie apart, each row tile's logits go ahead of the OTHER one's values, which is the
// order in which what they wait for is there when the two are half a tile apart.  (Asking for whichever can be made, by polling: 631
// instead of 513 us with 128 dimensions, where each product's start is on the critical path.)
template <class T>
struct Products {
  Smem& sm;
  const Abort& ab;
  uint32_t tmem, on;
  uint64_t q_desc, k_desc, v_desc;
  uint32_t done[2] = {0, 0}, asked[2] = {0, 0};          // products of either kind
  int with_tile[2] = {0, 0};
  uint32_t used = 0;                                     // tiles of the parts before
  uint32_t q_buf = 0;                                    // where this part's queries lie
  int n = 0, tiles = 0;                                  // of this part
  bool fine = true;

  __device__ __forceinline__ void wait(unsigned long long* bar, uint32_t parity) { fine = fine && mbar_wait_warp(smem_u32(bar), parity & 1u, ab); }

  __device__ __forceinline__ void ask(int x, int j) {
    if (j >= n || !fine) return;
    const uint32_t tile = used + (uint32_t)j, stage = tile % T::STAGES;
    if (x == 0) wait(&sm.k_full[stage], tile / T::STAGES);
    // the columns hold logits until they have been read, or the weights that the product before reads
    if (asked[x] > 0) wait(T::APART ? &sm.s_free[x] : &sm.o_done[x], asked[x] - 1);
    if (!fine) return;
    tc_fence_after();
    logits<T>(on, tmem + 128 * x, q_desc + (2 * q_buf + (uint32_t)x) * (T::QTILE >> 4), k_desc + stage * (T::KTILE >> 4));
    commit(on, smem_u32(&sm.s_full[x]));
    if (on) mbar_arrive(smem_u32(&sm.s_full[x]));         // hands on what this warp has seen: the tile's scales, the rows' factors
    ++asked[x];
    if (x == tiles - 1) {
      commit(on, smem_u32(&sm.k_empty[stage]));
      if (j + 1 == n) commit(on, smem_u32(&sm.q_free[q_buf]));
    }
  }
  __device__ __forceinline__ void add(int x, int j) {
    if (j < 0 || j >= n || !fine) return;
    const uint32_t tile = used + (uint32_t)j, stage = tile % T::STAGES;
    if (x == 0) wait(&sm.v_ready[stage], tile / T::STAGES);
    if (j == 0 && with_tile[x] > 0) wait(&sm.o_free[x], (uint32_t)(with_tile[x] - 1));
    wait(&sm.p_ready[x], done[x]);
    if (!fine) return;
    tc_fence_after();
    weigh<T>(on, tmem + T::O_COL + T::D * x, tmem + T::P_COL + T::P_STEP * x, v_desc + stage * (T::VTILE >> 4), j > 0 ? 1u : 0u);
    commit(on, smem_u32(&sm.o_done[x]));
    ++done[x];
    if (x == tiles - 1) commit(on, smem_u32(&sm.v_empty[stage]));
  }
};

template <class T>
__device__ __forceinline__ void issue_products(Smem& sm, uint32_t tmem, uint32_t q_tiles, uint32_t k_ring, uint32_t v_ring, const Abort& ab) {
  Products<T> p{sm, ab, tmem, elect_one() ? 1u : 0u, smem_desc<T::SPAN>(q_tiles), smem_desc<T::SPAN>(k_ring), value_desc(v_ring)};
  int n_parts = 0, with_keys = 0;
  for (;;) {
    p.wait(&sm.part_full[n_parts & 1], (uint32_t)(n_parts >> 1));
    if (!p.fine || sm.part[n_parts & 1].live <= 0) break;
    p.n = sm.part[n_parts & 1].n_tiles;
    p.tiles = sm.part[n_parts & 1].live > 128 ? 2 : 1;
    if (p.n > 0) {
      p.q_buf = (uint32_t)(with_keys % T::QBUFS);
      p.wait(&sm.q_ready[p.q_buf], (uint32_t)(with_keys / T::QBUFS));
      ++with_keys;
      if (!T::APART) {
#pragma unroll 1
        for (int j = -1; p.fine && j < p.n; ++j) {
          p.add(0, j);
          p.ask(0, j + 1);
          if (p.tiles == 2) {
            p.add(1, j);
            p.ask(1, j + 1);
          }
        }
      } else {
#pragma unroll 1
        for (int j = -1; p.fine && j <= p.n; ++j) {
          p.ask(0, j + 1);
          if (p.tiles == 2) {
            p.add(1, j - 1);
            p.ask(1, j + 1);
          }
          p.add(0, j);
        }
      }
      for (int x = 0; x < p.tiles; ++x) ++p.with_tile[x];
      p.used += (uint32_t)p.n;
      if (!p.fine) break;
    }
    __syncwarp();
    if (p.on) mbar_arrive(smem_u32(&sm.part_empty[n_parts & 1]));
    ++n_parts;
  }
  commit(p.on, smem_u32(&sm.mma_done));
  mbar_wait_warp(smem_u32(&sm.mma_done), 0u, ab);
}

// ---------------------------------------------------------------------------------------------- softmax and output
template <class T>
__device__ __forceinline__ void write_rows(const PromptArgs& args, const Part& p, int r, uint32_t o_addr, const RowStats& stats, bool any) {
  constexpr int D = T::D;
  const AttendArgs& a = args.a;
  const bool whole = (p.flags & kFromStart) && (p.flags & kToEnd), live = r < p.live;
  const uint32_t rr = (uint32_t)p.row_tile * kRows + (uint32_t)r;
  const int token = (int)(rr / (uint32_t)a.group), head = p.head * a.group + (int)(rr - (uint32_t)token * (uint32_t)a.group), slot = 2 * blockIdx.x + ((p.flags & kFromStart) ? 1 : 0);
  const int64_t row = p.row0 + token;
  const float inv = stats.l == 0.f ? 0.f : 1.f / stats.l, factor = output_factor<T::FP8>(stats);
  const int pos = p.pos0 + token, dirty = p.dirty;
#pragma unroll 1
  for (int c = 0; c < D; c += 32) {
    __syncwarp();
    uint32_t raw[32];
    if (any) {
      tmem_issue<32>(o_addr + c, raw);
      tmem_load_wait();
      tmem_ready<32>(raw);
    }
    float x[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) x[T::INT4 ? code_place(i) : i] = any ? __uint_as_float(raw[i]) : 0.f;
    if (dirty) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const bool nan = p.bad[0][c + i] <= pos, plus = p.bad[1][c + i] <= pos, minus = p.bad[2][c + i] <= pos;
        if (nan || (plus && minus)) x[i] = __int_as_float(0x7fffffff);
        else if (plus || minus) x[i] += plus ? INFINITY : -INFINITY;
      }
    }
    if (!live) {
      // a row that does not exist
    } else if (whole) {
      uint4* dst = reinterpret_cast<uint4*>(a.out.data + row * a.out.stride_row + head * a.out.stride_head + c);
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] = nan_if_infinite<T::FP8>(x[i]) * inv * factor;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        dst[i] = make_uint4(pack_bf16(x[8 * i], x[8 * i + 1]), pack_bf16(x[8 * i + 2], x[8 * i + 3]), pack_bf16(x[8 * i + 4], x[8 * i + 5]),
                            pack_bf16(x[8 * i + 6], x[8 * i + 7]));
    } else {
      float4* dst = reinterpret_cast<float4*>(args.parts.sums + ((int64_t)slot * kRows + r) * D + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) dst[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
  }
  if (!live) return;
  if (!whole) args.parts.stats[slot * kRows + r] = make_float4(stats.m, stats.m_sum, stats.l, 0.f);
  else if (a.lse != nullptr) a.lse[row * a.lse_stride_row + head * a.lse_stride_head] = row_lse(stats);
}

template <class T>
__device__ __forceinline__ void softmax_rows(const PromptArgs& args, Smem& sm, uint32_t tmem, const Abort& ab) {
  constexpr int D = T::D;
  const AttendArgs& a = args.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, x = warp >> 2;
  const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_addr = tmem + 128 * x + lanes, o_addr = tmem + T::O_COL + D * x + lanes,
                 p_addr = tmem + T::P_COL + T::P_STEP * x + lanes;
  const int r = x * 128 + (warp & 3) * 32 + lane;        // the thread's row of the part
  PartReader reader;
  int64_t seen = 0;                                      // tiles of this row tile
  int64_t info_at = 0;                                   // tiles of all parts
  while (Part* pp = reader.next(sm, ab)) {
    const Part& p = *pp;
    const bool mine = x * 128 < p.live;
    const int n = p.n_tiles;
    float m = kNoReference, m_sum = kNoReference, l = 0.f;   // m_sum: 8 bits
    if (mine && n > 0) {
      const int token = (int)(((uint32_t)p.row_tile * kRows + (uint32_t)r) / (uint32_t)a.group);
      const int hi = a.causal ? min(p.end, p.pos0 + token + 1) : p.end, first = p.first;
      float qf = 1.f;
      for (int j = 0; j < n; ++j, ++seen) {
        const int key0 = (p.tile0 + j) * kKeys;
        if (!mbar_wait_warp(smem_u32(&sm.s_full[x]), (uint32_t)seen & 1u, ab)) return;
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_issue<32>(s_addr + 32 * c, s[c]);
        float f[2], add[2];
        if constexpr (T::FP8) {
          const TileInfo& info = sm.info[(info_at + j) % kInfo];
          if (j == 0) qf = p.q_factor[r];
#pragma unroll
          for (int g = 0; g < 2; ++g) f[g] = logit_factor(info.k_scale[g], qf), add[g] = info.v_log2[g];
        } else {
#pragma unroll
          for (int g = 0; g < 2; ++g) f[g] = a.c, add[g] = 0.f;
        }
        tmem_load_wait();
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ready<32>(s[c]);
        if (__any_sync(0xffffffffu, key0 < first || key0 + kKeys > hi)) {
          const int lo_i = first - key0, hi_i = hi - key0;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (32 * c + i < lo_i || 32 * c + i >= hi_i) s[c][i] = 0xff800000u;
        }
        if constexpr (T::APART) {
          tc_fence_before();                             // the logits are in registers
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sm.s_free[x]));
        }
        // the row's largest logit (scales are positive); on the way through the exponentials below it would cost registers that
        // are not there (554 instead of 513 us)
        float top = -INFINITY, top_sum = -INFINITY;      // with the values' scales, and without
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 32; i += 2)
              t[(i >> 1) & 3] = max3(t[(i >> 1) & 3], __uint_as_float(s[2 * g + c][i]), __uint_as_float(s[2 * g + c][i + 1]));
          const float largest = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])) * f[g];
          top = fmaxf(top, largest + add[g]);
          top_sum = fmaxf(top_sum, largest);
        }
        auto above = [&](int g) { return above_weights(add[g] - m, m_sum); };
        bool over = T::FP8 ? top - m > kLazy + kShift : top > m + kLazy;
        if constexpr (T::FP8) over |= top_sum - m_sum > kLazy || above(0) > kFar || above(1) > kFar;
        if constexpr (T::APART) {
          // the weights go where the product with the tile before may still read
          if (seen > 0 && !mbar_wait_warp(smem_u32(&sm.o_done[x]), (uint32_t)(seen - 1) & 1u, ab)) return;
          tc_fence_after();
        }
        if (__any_sync(0xffffffffu, over)) {
          const float now = fmaxf(m, T::FP8 ? top - kShift : top), scale = fast_exp2(m - now);
          m = now;
          if constexpr (T::FP8) {
            const float now_sum = fmaxf(m_sum, top_sum);
            l *= fast_exp2(m_sum - now_sum);
            m_sum = now_sum;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              if (!__any_sync(0xffffffffu, above(g) > kFar)) continue;
              float own = 0.f;
#pragma unroll
              for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i) own += fast_exp2(fmaf(__uint_as_float(s[2 * g + c][i]), f[g], -m_sum));
              if (above(g) > kFar) l += own;
            }
          } else {
            l *= scale;
          }
          if (j > 0) {
            // the product with the tile before is done: it was waited for above, or before these logits' product
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              tmem_issue<16>(o_addr + c, o);
              tmem_load_wait();
              tmem_ready<16>(o);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * scale);
              tmem_store<16>(o_addr + c, o);
            }
          }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const uint64_t ff = pack2(f[g], f[g]), off = pack2(add[g] - m, add[g] - m);
          uint64_t sum[2] = {0ull, 0ull};
          uint32_t w[32];
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float u, v;
              unpack2(fma2(pack2(s[2 * g + c][i], s[2 * g + c][i + 1]), ff, off), u, v);
              u = fast_exp2(u);
              v = fast_exp2(v);
              sum[c] = add2(sum[c], pack2(u, v));
              w[16 * c + (i >> 1)] = T::FP8 ? pack_f16(u, v) : pack_bf16(u, v);
            }
          tmem_store<32>(p_addr + 32 * g, w);
          float u, v;
          unpack2(add2(sum[0], sum[1]), u, v);
          if constexpr (T::FP8) l = fmaf(u + v, above(g) > kFar ? 0.f : fast_exp2(above(g)), l);
          else l += u + v;
        }
        tmem_store_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.p_ready[x]));
      }
      if (!mbar_wait_warp(smem_u32(&sm.o_done[x]), (uint32_t)(seen - 1) & 1u, ab)) return;
      tc_fence_after();
    }
    if (mine) {
      if (!mbar_wait_warp(smem_u32(&sm.values_done[reader.n & 1]), (uint32_t)(reader.n >> 1) & 1u, ab)) return;
      write_rows<T>(args, p, r, o_addr, RowStats{m, T::FP8 ? m_sum : m, l}, n > 0);
      tc_fence_before();
      __syncwarp();
      if (n > 0 && lane == 0) mbar_arrive(smem_u32(&sm.o_free[x]));
    }
    if (threadIdx.x == 0 && (p.flags & kFromStart) && !(p.flags & kToEnd)) {
      args.parts.headers[2 * blockIdx.x] = make_int4(p.behind, p.row0, p.head, p.row_tile);
      args.parts.headers[2 * blockIdx.x + 1] = make_int4(p.live, 0, 0, 0);
    }
    info_at += n;
    reader.done(sm);
  }
}

// ---------------------------------------------------------------------------------------------- kernel
template <int D, int BITS>
__global__ void __launch_bounds__(kThreads, 1) attend_prompt_kernel(const __grid_constant__ PromptArgs args) {
  using T = Traits<D, BITS>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* q_tiles = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  unsigned char* k_ring = q_tiles + T::QBUFS * 2 * T::QTILE;
  unsigned char* v8_ring = k_ring + T::STAGES * T::KTILE;   // what is copied to be widened
  unsigned char* v_ring = v8_ring + T::STAGES * T::V8TILE + T::RAWS * 2 * T::RAW;
  Smem& sm = *reinterpret_cast<Smem*>(v_ring + T::STAGES * T::VTILE);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sm.s_full[i]), 2);
      mbar_init(smem_u32(&sm.s_free[i]), 4);
      mbar_init(smem_u32(&sm.p_ready[i]), 4);
      mbar_init(smem_u32(&sm.o_done[i]), 1);
      mbar_init(smem_u32(&sm.o_free[i]), 4);
      mbar_init(smem_u32(&sm.part_full[i]), 1);
      mbar_init(smem_u32(&sm.part_empty[i]), 13);        // warps 0-11 and the one that issues products
      mbar_init(smem_u32(&sm.values_done[i]), 4);
      mbar_init(smem_u32(&sm.q_ready[i]), 4);
      mbar_init(smem_u32(&sm.q_free[i]), 1);
    }
    mbar_init(smem_u32(&sm.mma_done), 1);
    for (int i = 0; i < T::STAGES; ++i) {
      mbar_init(smem_u32(&sm.k_full[i]), T::INT4 ? 4 : 1);
      mbar_init(smem_u32(&sm.k_empty[i]), 1);
      mbar_init(smem_u32(&sm.v_full[i]), 1);
      mbar_init(smem_u32(&sm.v_ready[i]), 4);
      mbar_init(smem_u32(&sm.v_empty[i]), 1);
      mbar_init(smem_u32(&sm.v8_empty[i]), 4);
      mbar_init(smem_u32(&sm.k4_full[i]), 1);
      mbar_init(smem_u32(&sm.k4_empty[i]), 4);
    }
    sm.abort = 0;
    args.parts.headers[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  find_start(args, sm);                                  // barriers of the CTA
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const int64_t total = sm.total, per = (total + gridDim.x - 1) / gridDim.x, w0 = per * blockIdx.x, w1 = min(w0 + per, total);
  grid_launch_dependents();
  const Abort ab{&sm.abort, args.a.dev_status};
  if (warp < 8) reg_inc<kSoftmaxRegs>();
  else reg_dec<kOtherRegs>();
  if (w0 < w1) {
    if (warp < 8) softmax_rows<T>(args, sm, tmem, ab);
    else if (warp < 12) prepare_values<T>(args.a, sm, q_tiles, k_ring, v8_ring, v_ring, ab);
    else if (warp == 12) copy_tiles<T>(args, sm, smem_u32(k_ring), smem_u32(BITS == 16 ? v_ring : v8_ring), w0, w1, per, ab);
    else if (warp == 13) issue_products<T>(sm, tmem, smem_u32(q_tiles), smem_u32(k_ring), smem_u32(v_ring), ab);
  }
  tc_fence_before();
  __syncthreads();
  if (sm.abort != 0) {
    // a wait ran out: what is still in flight gets time to land before the memory is given back
    const unsigned long long t0 = global_timer();
    while (global_timer() - t0 < 2000000ull) __nanosleep(1000);
  }
  __syncthreads();
  if (warp == 12) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int D, int BITS>
int32_t launch(const PromptArgs& args, int ctas, cudaStream_t stream) {
  using T = Traits<D, BITS>;
  static_assert(smem_bytes<T>() <= 227 * 1024);
  static ContextSet done;
  const int32_t st = allow_shared_memory(reinterpret_cast<const void*>(attend_prompt_kernel<D, BITS>), smem_bytes<T>(), done);
  if (st != SPF_OK) return st;
  attend_prompt_kernel<D, BITS><<<ctas, kThreads, smem_bytes<T>(), stream>>>(args);
  SPF_CUDA_CHECK(cudaGetLastError());
  return attend_join_launch(args.a, args.parts, kRows, kRows, D, T::FP8, ctas, stream);
}

}  // namespace

size_t attend_prompt_workspace_bytes(const spf_kv_cache* cache, int sm_count) { return parts_layout(kRows, cache->head_dim, sm_count).total; }

int32_t attend_prompt_launch(const AttendArgs& a, const spf_kv_cache* cache, int sm_count, void* workspace, cudaStream_t stream) {
  PromptArgs args{};
  args.a = a;
  args.parts = parts_at(workspace, kRows, cache->head_dim, sm_count);
  int32_t st = encode_pool_map("spf_attend", cache, cache->k_pool, kKeys, &args.k_map);
  if (st == SPF_OK) st = encode_pool_map("spf_attend", cache, cache->v_pool, kKeys, &args.v_map);
  if (st != SPF_OK) return st;
  const bool d64 = cache->head_dim == 64;
  switch (a.kv.bits) {
    case 4:
      st = encode_scale_map("spf_attend", cache, cache->k_scale, &args.k_scale_map);
      if (st == SPF_OK) st = encode_scale_map("spf_attend", cache, cache->v_scale, &args.v_scale_map);
      if (st != SPF_OK) return st;
      return d64 ? launch<64, 4>(args, sm_count, stream) : launch<128, 4>(args, sm_count, stream);
    case 8: return d64 ? launch<64, 8>(args, sm_count, stream) : launch<128, 8>(args, sm_count, stream);
    default: return d64 ? launch<64, 16>(args, sm_count, stream) : launch<128, 16>(args, sm_count, stream);
  }
}

}  // namespace spf
