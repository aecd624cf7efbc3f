// Attention of a step with few rows per key head (single tokens, lookahead tokens) over the paged cache, bf16, 8 or 4 bits.
//
//   z[r, s] = c q[r] . k[s]  (base-2 logits),   out[r] = sum_s 2^(z[r,s] - m_r) v[s] / l_r,   l_r = sum_s 2^(z[r,s] - m_r),
//   lse[r] = (m_r + log2 l_r) ln 2;   rows r = (new token i, head g of the key head's group), r = i G + g, in tiles of R.
//
// One pass over keys and values, each read once for all rows of a tile.  What bounds it is that read, so the work is dealt out
// by key tiles, not by sequences: the tiles of all (sequence, row tile, key head) triples, 64 or 128 keys each, form one list, and CTA
// c takes its c-th part, wherever that begins and ends.  A triple that one CTA has from end to end is written at once; one that
// several share leaves partial sums in the workspace, and a second kernel (launched behind the first without waiting for the
// host) joins them in the order of the keys.  All of it is worked out on the device from the lengths there.
//
// A CTA: one warp copies tiles into a ring (TMA, a tile's keys and their values a stage) and runs ahead across the triples' borders;
// four warps compute, each on its own 16 or 32 keys of every tile (many rows: some of the rows and more of the keys), with maxima, sums
// and outputs of their own in registers, so that nothing is exchanged between them until a triple ends.  Products are warp-level, with
// the keys (then the dimensions of the values) as the 16 rows of the left operand and the query rows as the 8 columns of the right
// one: a single token's few heads fill a product, where they would be half or less of the left operand's rows, and the tensor
// cores' big instruction would be idle for the most part; the keys' read takes longer than these.  Logits have keys as
// rows and queries as columns; a weight is wanted the other way round, which one movmatrix per 8 x 8 does.
//
// The reference m_r moves only when a logit exceeds it by 8 (2^8 is far from any format's limit): most tiles need no exchange
// of maxima and no rescaling of the output.  Weights are rounded to the format of the second product's operands, fp16 (11 bits) over
// 8-bit values, bf16 (8 bits; the output is bf16 too) over bf16 ones; their sum l is taken in fp32 before that.  Up to 8 rows over a bf16
// cache, where the read leaves time, weights are two bf16 terms (off by 2^-16): 16 sequences of 4 to 32k tokens take 172 us with either
// one or two, one short prompt 11.2 instead of 10.8.  Two terms would cost 32 rows 8 % (64 dimensions, bf16) and 8-bit caches 16 %.
//
// 8 bits, keys: multiplied as they are (m16n8k32, E4M3) by queries in two terms, E4M3 and E5M2: q 2^e = hi + lo, with the power of
// two e of a row that takes its largest element to (224, 448].  Exact for elements within 2^13 of that one, off by at most 2^-21 of
// it below: hi has 4 significant bits, what it leaves is at most half its step and fits lo's 3.
// 8 bits, values: widened to fp16, exactly, next to the products (widen4; both operands by the conversion instruction, which is
// slow: 697 instead of 384 us for four sequences of 131 to 250 thousand tokens).  A tile's value scale s_v joins its logits, so that the
// weights are p s_v / (the largest such so far) and never leave fp16's range; their sum l has a reference of its own (RowStats):
//   z'[r,s] = z[r,s] + log2 s_v,  w = 2^(z' - m'),  l = sum 2^(z - m),  out = 2^(m' - m) sum w byte / l,  lse = (m + log2 l) ln 2.
// m' lies 7 below the largest z' seen (but for the 8 above), which leaves small weights more of fp16's range.
//
// 4 bits: an element is s (code - 8), a scale for 32 dimensions of a token.  Widening them would take more instructions than the read of half as many
// bytes leaves room for, so codes are multiplied without being converted: the four bits of a code in the lowest (or the next) four of a bf16 number's
// are code 2^-133 (16 times that), a subnormal number, which the products take exactly; one instruction makes two of them.  The 8 is taken
// off the sums: of 32 keys' elements by where the sum starts, of values by a product with eights in the codes' places.  Scales of keys multiply
// the sums of their 32 dimensions, those of values the weights.  Powers of two in the queries, and in the reference of the weights, which
// lies 2^64 below the largest, keep all sums in fp32's normal range.  32 sequences of up to 16k tokens, 8 heads of 128 dimensions, one token each:
// 77 us, where the bytes take 49 (8 bits: 111, 88), and 58 without products; four of 131 to 250 thousand 189 (150).  What the rest goes to: the
// chain of a warp's tile, of which three a scheduler run at a time at 128 registers (four at 96 spill: 93 us).
//
// Keys that no row may see (behind the sequence's end, before its first key) take part with logits of -inf and values of zero,
// whatever the pool holds there.  Keys that only later rows of the step may see have weight zero; if their values are not
// finite, the tile's second product is made row by row, so that they reach the rows that see them and no others.
#include <algorithm>

#include "attend_step.cuh"

namespace spf {
namespace {

struct StepArgs {
  AttendArgs a;
  CUtensorMap k_map, v_map;
  CUtensorMap k_scale_map, v_scale_map;   // 4 bits
  AttendParts parts;
};

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// ---------------------------------------------------------------------------------------------- the list of tiles
template <class T>
__device__ __forceinline__ int tiles_of(const SeqSpan& s) { return max((s.end + T::KEYS - 1) / T::KEYS - s.first / T::KEYS, 1); }
template <class T>
__device__ __forceinline__ int row_tiles_of(const AttendArgs& a, const SeqSpan& s) {
  return (int)(((int64_t)s.n_new * a.group + T::R - 1) / T::R);
}
template <class T>
__device__ __forceinline__ int64_t cost_of(const AttendArgs& a, int b) {
  const SeqSpan s = seq_span(a, b);
  return (int64_t)row_tiles_of<T>(a, s) * a.kv.n_kv_heads * tiles_of<T>(s);
}

// Length of the list, and the sequence that holds the CTA's first tile.  Every thread sums up a run of sequences.
template <class T>
__device__ __forceinline__ void find_start(const StepArgs& args, SmallSmem& sm) {
  const AttendArgs& a = args.a;
  const int run = (a.step.n_seqs + T::THREADS - 1) / T::THREADS, lo = min((int)threadIdx.x * run, a.step.n_seqs), hi = min(lo + run, a.step.n_seqs);
  int64_t mine = 0;
  for (int b = lo; b < hi; ++b) mine += cost_of<T>(a, b);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t upto = mine;                                   // sum over the threads up to this one
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sm.scan[warp] = upto;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < T::THREADS / 32; ++w) {
    if (w < warp) upto += sm.scan[w];
    total += sm.scan[w];
  }
  const int64_t w0 = (total + gridDim.x - 1) / gridDim.x * blockIdx.x;
  if (threadIdx.x == 0) sm.total = total;
  if (w0 >= upto - mine && w0 < upto) {
    int64_t base = upto - mine;
    int b = lo;
    for (; b < hi - 1; ++b) {
      const int64_t c = cost_of<T>(a, b);
      if (w0 < base + c) break;
      base += c;
    }
    sm.start_seq = b;
    sm.start_base = base;
  }
  __syncthreads();
}

// The copying warp.  Each lane works out one of the next 32 tiles (block table, scales: loads in parallel), then the tiles are
// put into the ring one by one.
template <class T>
__device__ __forceinline__ void copy_tiles(const StepArgs& args, SmallSmem& sm, uint32_t ring, int64_t w0, int64_t w1, int64_t per, const Abort& ab) {
  const AttendArgs& a = args.a;
  const int lane = threadIdx.x & 31;
  const int64_t pool_rows = a.kv.n_blocks * a.kv.n_kv_heads * a.kv.block_tokens;
  int seq = sm.start_seq;
  int64_t base = sm.start_base;
  int stage = 0;
  int64_t issued = 0;
  uint32_t parity = 1;                                    // the ring's stages start out empty
  for (int64_t w = w0; w < w1; w += 32) {
    const int64_t mine = w + lane;
    TileDesc d{};
    int row = 0;
    if (mine < w1) {
      SeqSpan s = seq_span(a, seq);
      int tiles = tiles_of<T>(s), row_tiles = row_tiles_of<T>(a, s);
      int64_t cost = (int64_t)row_tiles * a.kv.n_kv_heads * tiles;
      while (mine >= base + cost && seq < a.step.n_seqs - 1) {
        base += cost;
        s = seq_span(a, ++seq);
        tiles = tiles_of<T>(s);
        row_tiles = row_tiles_of<T>(a, s);
        cost = (int64_t)row_tiles * a.kv.n_kv_heads * tiles;
      }
      const int64_t in_seq = mine - base, triple = in_seq / tiles;
      const int tile = (int)(in_seq - triple * tiles);
      const int64_t from = base + triple * tiles, to = from + tiles;      // the triple's place in the list
      d.row0 = s.row0;
      d.n_new = s.n_new;
      d.pos0 = s.pos0;
      d.first = s.first;
      d.end = s.end;
      d.head = (int)(triple / row_tiles);
      d.row_tile = (int)(triple - (int64_t)d.head * row_tiles);
      d.key0 = (s.first / T::KEYS + tile) * T::KEYS;
      d.flags = (mine == max(from, w0) ? kFirst : 0) | (mine == min(to, w1) - 1 ? kLast : 0) | (s.first >= s.end ? kNoKeys : 0) |
                (from >= w0 ? kFromStart : 0) | (to <= w1 ? kToEnd : 0) | ((int)((to - 1) / per - blockIdx.x) << 8);
      if (s.first < s.end) {
        row = pool_row(a, seq, d.head, d.key0);
        if constexpr (T::FP8) {
#pragma unroll
          for (int g = 0; g < T::KEYS / kScaleTokens; ++g) {
            const int key = d.key0 + g * kScaleTokens, at = row + g * kScaleTokens;
            d.k_scale[g] = a.c * group_scale(a.kv.k_scale, s, key, at, pool_rows);
            d.v_log2[g] = log2f(group_scale(a.kv.v_scale, s, key, at, pool_rows));
          }
        }
      }
    }
    const int count = (int)min((int64_t)32, w1 - w);
    for (int j = 0; j < count; ++j) {
      if (!mbar_wait_warp(smem_u32(&sm.empty[stage]), parity, ab)) {
        // a stage's last copy was its (issued - stage) / STAGES-th, rounded up
        if (lane < T::STAGES && issued > lane)
          drain_copy(smem_u32(&sm.full[lane]), (uint32_t)((issued - lane + T::STAGES - 1) / T::STAGES - 1) & 1u);
        return;
      }
      ++issued;
      if (lane == j) {
        sm.desc[stage] = d;
        const uint32_t bar = smem_u32(&sm.full[stage]), at = ring + stage * T::STAGE;
        if (d.flags & kNoKeys) {
          mbar_arrive(bar);
        } else {
          mbar_expect_tx(bar, T::STAGE);
          tma_load_3d(at, &args.k_map, 0, row, 0, bar);
          tma_load_3d(at + T::TILE, &args.v_map, 0, row, 0, bar);
          if constexpr (T::INT4) {
            tma_load_2d(at + 2 * T::TILE, &args.k_scale_map, 0, row / 128, bar);
            tma_load_2d(at + 2 * T::TILE + T::SCALES, &args.v_scale_map, 0, row / 128, bar);
          }
        }
      }
      if (++stage == T::STAGES) stage = 0, parity ^= 1;
    }
    seq = __shfl_sync(0xffffffffu, seq, count - 1);
    base = __shfl_sync(0xffffffffu, base, count - 1);
  }
}

// ---------------------------------------------------------------------------------------------- the computing warps
// Barrier of the computing warps (bounded, as every wait here).
struct Join {
  uint32_t bar, parity;
  __device__ __forceinline__ bool wait(const Abort& ab) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
    const bool ok = mbar_wait_warp(bar, parity, ab);
    parity ^= 1;
    return ok;
  }
};

// 16 dimensions of the values of 16 keys as the left operand: a[0], a[2] dimensions 0-7, a[1], a[3] 8-15.  The halves of a register
// are two keys (value_key).  8 bits: two such, for the 16 dimensions behind as well; 4 bits: two such of 32 dimensions that share scales, rows
// 0-7 the even dimensions, 8-15 the odd ones.
template <class T>
__device__ __forceinline__ void value_operand(uint32_t v_tile, int key, int mt, int lane, uint32_t (&a)[T::FP8 ? 2 : 1][4]) {
  static_assert(!T::INT4);
  if constexpr (T::FP8) {
    uint32_t r[4];
    // two 16 x 16 byte matrices, transposed: r[0] the four keys 4 c ... of dimension lane / 4, r[1] of the one 8 behind it
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(v_tile + tile_chunk<T>(key + (lane & 15), mt + (lane >> 4))));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      widen4(r[2 * i], a[i][0], a[i][2]);
      widen4(r[2 * i + 1], a[i][1], a[i][3]);
    }
  } else {
    ldsm4_t(v_tile + tile_chunk<T>(key + (lane >> 4) * 8 + (lane & 7), 2 * mt + ((lane >> 3) & 1)), a[0]);
  }
}
// The two keys in register e of a value operand.
template <class T>
__device__ __forceinline__ int value_key(int lane, int e, int half) {
  return T::FP8 ? 4 * (lane & 3) + (e >> 1) + 2 * half : 2 * (lane & 3) + half + 8 * (e >> 1);
}

// Zeroes the halves of an operand register whose keys lie outside [lo, hi).
__device__ __forceinline__ uint32_t keep_keys(uint32_t pair, int key_low, int key_high, int lo, int hi) {
  uint32_t mask = 0;
  if (key_low >= lo && key_low < hi) mask |= 0x0000ffffu;
  if (key_high >= lo && key_high < hi) mask |= 0xffff0000u;
  return pair & mask;
}
template <bool FP8>
__device__ __forceinline__ bool not_finite(uint32_t pair) {
  constexpr uint32_t kExp = FP8 ? 0x7c00u : 0x7f80u;
  return (pair & kExp) == kExp || ((pair >> 16) & kExp) == kExp;
}

// What a warp has of a triple: outputs (dimensions lane / 4 and 8 behind it of every 16, query rows 2 (lane % 4) and the next of
// every 8), references and sums of its rows.
template <class T>
struct State {
  float o[T::D / 16][T::NT][4];
  float eight[T::INT4 ? T::PARTS : 1][T::INT4 ? T::NT : 1][4];   // 4 bits: what 8 in place of the codes would give
  float m[T::NT][2], l[T::NT][2];
  float m_sum[T::FP8 ? T::NT : 1][2];                    // 8 bits
};

// Keys of a triple that its rows see: [first, end) that some do, below `all` that every one does.
struct Seen {
  int first, end, all;
};

// out += values . weights of the warp's keys from `key` (of the tile, which begins at key0) on, p[t][kt][nt] being a term of the weights
// of sixteen keys and eight rows.  GUARD: the tile has keys outside [first, end), whose values are taken as zeros.
template <class T, bool GUARD>
__device__ __forceinline__ void add_values(State<T>& st, const uint32_t (&p)[T::WTERMS][T::KT][T::NT][2], uint32_t v_tile, int key, int key0, const Seen& seen,
                                           int lane) {
  constexpr int kStep = T::FP8 ? 2 : 1;
#pragma unroll
  for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
    for (int m0 = 0; m0 < T::D / 16; m0 += kStep) {
      uint32_t v[kStep][4];
      value_operand<T>(v_tile, key + kt * 16, m0, lane, v);
      if (GUARD) {
        const int base = key0 + key + kt * 16;
#pragma unroll
        for (int i = 0; i < kStep; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[i][e] = keep_keys(v[i][e], base + value_key<T>(lane, e, 0), base + value_key<T>(lane, e, 1), seen.first, seen.end);
      }
#pragma unroll
      for (int i = 0; i < kStep; ++i)
#pragma unroll
        for (int nt = 0; nt < T::NT; ++nt)
#pragma unroll
          for (int t = 0; t < T::WTERMS; ++t) mma16<T::FP8>(st.o[m0 + i][nt], v[i], p[t][kt][nt][0], p[t][kt][nt][1]);
    }
}

// Codes of 16 keys' values in two times 32 dimensions, transposed: w[2 i] the four keys of rows 4 c ... and byte lane / 4, w[2 i + 1] of the
// byte 8 behind it.
template <class T>
__device__ __forceinline__ void code_operand(uint32_t v_tile, int key, int m0, int lane, uint32_t (&w)[4]) {
  const int r = lane & 15;
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
               : "r"(v_tile + tile_chunk<T>(key + operand_key<T>(2 * (r >> 2) + ((r >> 1) & 1), r & 1), m0 + (lane >> 4))));
}
// The products of 32 dimensions' codes, two words, and of eights in their places.
template <class T>
__device__ __forceinline__ void multiply_codes(State<T>& st, uint32_t w0, uint32_t w1, int part, int nt, const uint32_t (&p)[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t word = j ? w1 : w0;
    const uint32_t codes[4] = {word & 0x000f000fu, word & 0x00f000f0u, (word >> 8) & 0x000f000fu, (word >> 8) & 0x00f000f0u};
    mma16<false>(st.o[2 * part + j][nt], codes, p[0], p[1]);
  }
  const uint32_t eights[4] = {0x00080008u, 0x00800080u, 0x00080008u, 0x00800080u};
  mma16<false>(st.eight[part][nt], eights, p[0], p[1]);
}

// 4 bits: out += scales . codes . weights.  Codes are multiplied as subnormal numbers, as those of the keys are (tile_logits); scales go into
// the weights, and 8 times the sum of these is subtracted at the triple's end.  x[kt][nt][h]: the weights in fp32.
//
// Weights are rounded to bf16 and turned as they are, once for all scales, and multiplied by pairs of scales as bf16 pairs, which rounds them
// again (both together off by up to 2^-8); scaled in fp32 first, each scale would have a rounding, a packing and a turn of its own, 28
// instructions a sixteen of keys more.  Where some keys are not seen by some rows (add_some_codes) that is what is done:
// values of keys that a row does not see count as zeros, whatever their scales.
template <class T>
__device__ __forceinline__ void add_codes(State<T>& st, const float (&x)[T::KT][T::NT][2][2], uint32_t v_tile, uint32_t scales, int key, int lane) {
#pragma unroll
  for (int kt = 0; kt < T::KT; ++kt) {
    // scales of the two keys in a register of the right operand, rows 2 c and 2 c + 1 of either half: neighbours
    uint32_t pairs[2][T::PARTS];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = key + kt * 16 + operand_key<T>(2 * (lane & 3), h);
      uint32_t w[T::PARTS];
      if constexpr (T::PARTS == 4) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(scales + at * 8));
      else asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(scales + at * 4));
#pragma unroll
      for (int p = 0; p < T::PARTS; ++p) pairs[h][p] = __byte_perm(w[p / 2], w[T::PARTS / 2 + p / 2], p & 1 ? 0x7632 : 0x5410);
    }
    uint32_t turned[T::NT][2];
#pragma unroll
    for (int nt = 0; nt < T::NT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) turned[nt][h] = transpose8(pack_bf16(x[kt][nt][h][0], x[kt][nt][h][1]));
#pragma unroll
    for (int m0 = 0; m0 < T::PARTS; m0 += 2) {
      uint32_t w[4];
      code_operand<T>(v_tile, key + kt * 16, m0, lane, w);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int part = m0 + i;
#pragma unroll
        for (int nt = 0; nt < T::NT; ++nt) {
          uint32_t p[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(p[h]) : "r"(turned[nt][h]), "r"(pairs[h][part]));
          multiply_codes<T>(st, w[2 * i], w[2 * i + 1], part, nt, p);
        }
      }
    }
  }
}
template <class T>
__device__ __forceinline__ void add_some_codes(State<T>& st, const float (&x)[T::KT][T::NT][2][2], const int (&sees)[T::NT][2], uint32_t v_tile, uint32_t scales, int key,
                                          int key0, int first, int lane) {
#pragma unroll
  for (int kt = 0; kt < T::KT; ++kt) {
    float s[2][T::PARTS];
#pragma unroll
    for (int h = 0; h < 2; ++h) load_scales<T>(scales, key + kt * 16 + key_of<T>(lane, h), s[h]);
#pragma unroll
    for (int m0 = 0; m0 < T::PARTS; m0 += 2) {
      uint32_t w[4];
      code_operand<T>(v_tile, key + kt * 16, m0, lane, w);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int part = m0 + i;
#pragma unroll
        for (int nt = 0; nt < T::NT; ++nt) {
          uint32_t p[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float u = x[kt][nt][h][0] * s[h][part], v = x[kt][nt][h][1] * s[h][part];
            const int at = key0 + key + kt * 16 + key_of<T>(lane, h);
            if (at < first || at >= sees[nt][0]) u = 0.f;
            if (at < first || at >= sees[nt][1]) v = 0.f;
            p[h] = transpose8(pack_bf16(u, v));
          }
          multiply_codes<T>(st, w[2 * i], w[2 * i + 1], part, nt, p);
        }
      }
    }
  }
}

// Whether the warp has values that are not finite of keys that some row sees and others do not.
template <class T>
__device__ __noinline__ bool odd_values(uint32_t v_tile, int key, int key0, int all, int end, int lane) {
  constexpr int kStep = T::FP8 ? 2 : 1;
  bool odd = false;
  for (int kt = 0; kt < T::KT; ++kt)
    for (int m0 = 0; m0 < T::D / 16; m0 += kStep) {
      uint32_t v[kStep][4];
      value_operand<T>(v_tile, key + kt * 16, m0, lane, v);
      const int base = key0 + key + kt * 16;
#pragma unroll
      for (int i = 0; i < kStep; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          odd |= not_finite<T::FP8>(keep_keys(v[i][e], base + value_key<T>(lane, e, 0), base + value_key<T>(lane, e, 1), all, end));
    }
  return __any_sync(0xffffffffu, odd);
}

// add_values where there are such: row by row, each with the values that it sees.
template <class T>
__device__ __forceinline__ void add_odd_values(State<T>& st, const uint32_t (&p)[T::WTERMS][T::KT][T::NT][2], uint32_t v_tile, int key, int key0, const Seen& seen,
                                               const TileDesc& d, int group, int causal, int row_in_triple, int lane) {
  constexpr int kStep = T::FP8 ? 2 : 1;
#pragma unroll 1
  for (int r = 0; r < 8; ++r) {
    const bool mine = (lane >> 2) == r;
#pragma unroll
    for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
      for (int m0 = 0; m0 < T::D / 16; m0 += kStep) {
        uint32_t v[kStep][4];
        value_operand<T>(v_tile, key + kt * 16, m0, lane, v);
        const int base = key0 + key + kt * 16;
#pragma unroll
        for (int nt = 0; nt < T::NT; ++nt) {
          const int hi = causal ? min(seen.end, d.pos0 + (row_in_triple + nt * 8 + r) / group + 1) : seen.end;
#pragma unroll
          for (int i = 0; i < kStep; ++i) {
            float part[4] = {0.f, 0.f, 0.f, 0.f};
            uint32_t vr[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) vr[e] = keep_keys(v[i][e], base + value_key<T>(lane, e, 0), base + value_key<T>(lane, e, 1), seen.first, hi);
#pragma unroll
            for (int t = 0; t < T::WTERMS; ++t) mma16<T::FP8>(part, vr, mine ? p[t][kt][nt][0] : 0u, mine ? p[t][kt][nt][1] : 0u);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (2 * (lane & 3) + (e & 1) == r) st.o[m0 + i][nt][e] += part[e];
          }
        }
      }
  }
}

template <class T>
__device__ __forceinline__ void compute_tiles(const StepArgs& args, SmallSmem& sm, unsigned char* ring_ptr, uint32_t ring, unsigned char* q_tile,
                                              int64_t w0, int64_t n_tiles, const Abort& ab) {
  constexpr int D = T::D, R = T::R, NT = T::NT, KT = T::KT;
  // 4 bits: the reference lies 2^64 below the largest weight, so that codes of 2^-133 times weights and scales make normal numbers
  constexpr float kBelow = T::INT4 ? 64.f : 0.f;
  const AttendArgs& a = args.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row_off = warp % T::WR * NT * 8, key_warp = warp / T::WR, key_off = key_warp * T::KW;
  const uint32_t q_addr = smem_u32(q_tile);
  __shared__ QueryNotes<T> notes;
  Join join{smem_u32(&sm.join), 0};
  State<T> st;
  int sees[NT][2];                                       // the key behind the last one that a row sees
  Seen seen{0, 0, 0};
  Queries<T> queries;
  int stage = 0;
  uint32_t parity = 0;
  {
    // the queries of the CTA's first triple, while its first keys are on their way
    const SeqSpan s = seq_span(a, sm.start_seq);
    const int64_t triple = (w0 - sm.start_base) / tiles_of<T>(s);
    TileDesc d;
    d.row0 = s.row0, d.n_new = s.n_new;
    d.head = (int)(triple / row_tiles_of<T>(a, s));
    d.row_tile = (int)(triple - (int64_t)d.head * row_tiles_of<T>(a, s));
    load_queries<T>(a, d, q_tile, notes);
  }
  for (int64_t tile = 0; tile < n_tiles; ++tile) {
    if (!mbar_wait_warp(smem_u32(&sm.full[stage]), parity, ab)) return;
    const TileDesc& d = sm.desc[stage];
    const int flags = d.flags;
    if (flags & kFirst) {
      if (tile > 0) load_queries<T>(a, d, q_tile, notes);
      if (!join.wait(ab)) return;
      const int row_first = d.row_tile * R;
      seen.first = d.first, seen.end = d.end;
      seen.all = a.causal ? min(d.end, d.pos0 + row_first / a.group + 1) : d.end;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = row_first + row_off + nt * 8 + 2 * (lane & 3) + e;
          sees[nt][e] = a.causal ? min(d.end, d.pos0 + row / a.group + 1) : d.end;
          st.m[nt][e] = kNoReference;
          st.l[nt][e] = 0.f;
          if constexpr (T::FP8) st.m_sum[nt][e] = kNoReference;
        }
#pragma unroll
        for (int m = 0; m < D / 16; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) st.o[m][nt][e] = 0.f;
      }
      if constexpr (T::INT4) {
#pragma unroll
        for (int p = 0; p < T::PARTS; ++p)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) st.eight[p][nt][e] = 0.f;
      }
      queries.load(q_addr, notes, row_off, lane);
    }
    if (!(flags & kNoKeys)) {
      const uint32_t k_tile = ring + stage * T::STAGE, v_tile = k_tile + T::TILE;
      const int key0 = d.key0, group64 = T::KEYS > kScaleTokens ? key_off / kScaleTokens : 0;
      const bool guard = key0 < seen.first || key0 + T::KEYS > seen.all;
      // logits of the warp's keys and rows
      float z[KT][NT][4];
      tile_logits<T>(z, queries, q_addr, row_off, k_tile, k_tile + 2 * T::TILE, key_off, lane);
      if (guard) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int key = key0 + key_off + kt * 16 + key_of<T>(lane, e >> 1);
              if (key < seen.first || key >= sees[nt][e & 1]) z[kt][nt][e] = -INFINITY;
            }
      }
      // base-2 logits are z f + add; the largest decides whether a row's reference moves
      const float add = T::FP8 ? d.v_log2[group64] : 0.f, k_scale = T::FP8 ? d.k_scale[group64] : a.c;
      float f[NT][2], top[NT][2];
      auto offset = [&](int nt, int e) { return add - st.m[nt][e]; };
      bool over = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          f[nt][e] = T::FP8 ? logit_factor(k_scale, queries.factor[nt][e]) : T::INT4 ? queries.factor[nt][e] : k_scale;
          float t = fmaxf(z[0][nt][e], z[0][nt][2 + e]);
#pragma unroll
          for (int kt = 1; kt < KT; ++kt) t = max3(t, z[kt][nt][e], z[kt][nt][2 + e]);
          top[nt][e] = t * f[nt][e];
          if constexpr (T::FP8) {
            const float off = offset(nt, e);
            over |= top[nt][e] + off > kLazy + kShift || top[nt][e] - st.m_sum[nt][e] > kLazy || above_weights(off, st.m_sum[nt][e]) > kFar;
          } else {
            over |= top[nt][e] > st.m[nt][e] + (kLazy + kBelow);
          }
        }
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float largest = top[nt][e];
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, o));
            const float m = fmaxf(st.m[nt][e], T::FP8 ? largest + add - kShift : largest - kBelow), scale = fast_exp2(st.m[nt][e] - m);
            st.m[nt][e] = m;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) st.o[i][nt][e] *= scale, st.o[i][nt][2 + e] *= scale;
            if constexpr (T::INT4) {
#pragma unroll
              for (int p = 0; p < T::PARTS; ++p) st.eight[p][nt][e] *= scale, st.eight[p][nt][2 + e] *= scale;
            }
            if constexpr (T::FP8) {
              const float m_sum = fmaxf(st.m_sum[nt][e], largest);
              st.l[nt][e] *= fast_exp2(st.m_sum[nt][e] - m_sum);
              st.m_sum[nt][e] = m_sum;
              if (above_weights(offset(nt, e), m_sum) > kFar) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                  for (int h = 0; h < 2; ++h) st.l[nt][e] += fast_exp2(fmaf(z[kt][nt][2 * h + e], f[nt][e], -m_sum));
              }
            } else {
              st.l[nt][e] *= scale;
            }
          }
      }
      uint32_t p[T::WTERMS][KT][NT][2];                  // not for 4 bits
      float weight[T::INT4 ? KT : 1][NT][2][2];          // 4 bits
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float off[2], sum[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 2; ++e) off[e] = offset(nt, e);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float x = fast_exp2(fmaf(z[kt][nt][2 * h], f[nt][0], off[0])), y = fast_exp2(fmaf(z[kt][nt][2 * h + 1], f[nt][1], off[1]));
            sum[0] += x;
            sum[1] += y;
            if constexpr (T::INT4) {
              weight[kt][nt][h][0] = x, weight[kt][nt][h][1] = y;
              continue;
            }
            const uint32_t w = T::FP8 ? pack_f16(x, y) : pack_bf16(x, y);
            p[0][kt][nt][h] = transpose8(w);
            if constexpr (T::WTERMS == 2) p[1][kt][nt][h] = transpose8(pack_bf16(x - __uint_as_float(w << 16), y - __uint_as_float(w & 0xffff0000u)));
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if constexpr (T::FP8) {
            const float above = above_weights(off[e], st.m_sum[nt][e]);
            st.l[nt][e] = fmaf(sum[e], above > kFar ? 0.f : fast_exp2(above), st.l[nt][e]);
          } else {
            st.l[nt][e] += sum[e];
          }
        }
      }
      if constexpr (T::INT4) {
        const uint32_t v_scales = k_tile + 2 * T::TILE + T::SCALES;
        if (!guard) add_codes<T>(st, weight, v_tile, v_scales, key_off, lane);
        else add_some_codes<T>(st, weight, sees, v_tile, v_scales, key_off, key0, seen.first, lane);
      } else if (!guard) add_values<T, false>(st, p, v_tile, key_off, key0, seen, lane);
      else if (seen.all >= seen.end || !odd_values<T>(v_tile, key_off, key0, seen.all, seen.end, lane)) add_values<T, true>(st, p, v_tile, key_off, key0, seen, lane);
      else add_odd_values<T>(st, p, v_tile, key_off, key0, seen, d, a.group, a.causal, d.row_tile * R + row_off, lane);
    }
    if (flags & kLast) {
      if constexpr (T::INT4) {
        // codes less 8, and both powers of two taken out: of the codes' places and of the reference
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int m = 0; m < D / 16; ++m) st.o[m][nt][e] = (st.o[m][nt][e] - st.eight[m / 2][nt][e]) * (e < 2 ? 0x1p69f : 0x1p65f);
#pragma unroll
          for (int e = 0; e < 2; ++e) st.l[nt][e] *= 0x1p-64f, st.m[nt][e] += kBelow;
        }
      }
      // the warps' sums of a row, each against its own reference
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float l = st.l[nt][e];
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
          if (lane < 4) sm.stats[key_warp][row_off + nt * 8 + 2 * lane + e] = RowStats{st.m[nt][e], T::FP8 ? st.m_sum[nt][e] : st.m[nt][e], l};
        }
      if (!join.wait(ab)) return;                        // statistics are there, and the stage's tile is read
      float f[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = row_off + nt * 8 + 2 * (lane & 3) + e;
          float top = kNoReference;
#pragma unroll
          for (int w = 0; w < T::WK; ++w) top = fmaxf(top, sm.stats[w][r].m);
          f[nt][e] = fast_exp2(st.m[nt][e] - top);
        }
      const bool whole = (flags & kFromStart) && (flags & kToEnd);
      const int slot = 2 * blockIdx.x + ((flags & kFromStart) ? 1 : 0);
      const int live = min(R, d.n_new * a.group - d.row_tile * R);
      float* buf = reinterpret_cast<float*>(ring_ptr + stage * T::STAGE);
      constexpr int kSwizzle = (T::JOIN / 8 < 4 ? T::JOIN / 8 : 4) - 1;      // rows 2 c share a bank otherwise
#pragma unroll 1
      for (int c0 = 0; c0 < D; c0 += T::JOIN) {
#pragma unroll
        for (int m = 0; m < D / 16; ++m) {
          if (16 * m < c0 || 16 * m >= c0 + T::JOIN) continue;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = row_off + nt * 8 + 2 * (lane & 3) + (e & 1), col = 16 * m - c0 + (T::INT4 ? 2 * (lane >> 2) + (e >> 1) : (lane >> 2) + 8 * (e >> 1));
              buf[(key_warp * R + r) * T::JOIN + (col ^ (((r >> 1) & kSwizzle) << 3))] = st.o[m][nt][e] * f[nt][e & 1];
            }
        }
        if (!join.wait(ab)) return;
        for (int item = threadIdx.x; item < live * (T::JOIN / 8); item += kWarps * 32) {
          const int r = item / (T::JOIN / 8), col = item % (T::JOIN / 8) * 8, at = col ^ (((r >> 1) & kSwizzle) << 3);
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
          for (int w = 0; w < T::WK; ++w) {
            const float4* src = reinterpret_cast<const float4*>(buf + (w * R + r) * T::JOIN + at);
            const float4 u = src[0], v = src[1];
            x[0] += u.x, x[1] += u.y, x[2] += u.z, x[3] += u.w, x[4] += v.x, x[5] += v.y, x[6] += v.z, x[7] += v.w;
          }
          RowStats all{kNoReference, kNoReference, 0.f};
#pragma unroll
          for (int w = 0; w < T::WK; ++w) all.m = fmaxf(all.m, sm.stats[w][r].m), all.m_sum = fmaxf(all.m_sum, sm.stats[w][r].m_sum);
#pragma unroll
          for (int w = 0; w < T::WK; ++w) all.l += sm.stats[w][r].l * fast_exp2(sm.stats[w][r].m_sum - all.m_sum);
          if (whole) {
            const int rr = d.row_tile * R + r;
            const int64_t row = d.row0 + rr / a.group;
            const int head = d.head * a.group + rr % a.group;
            const float inv = all.l == 0.f ? 0.f : 1.f / all.l, factor = output_factor<T::FP8>(all);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = nan_if_infinite<T::FP8>(x[i]) * inv * factor;
            uint4 v;
            v.x = pack_bf16(x[0], x[1]), v.y = pack_bf16(x[2], x[3]);
            v.z = pack_bf16(x[4], x[5]), v.w = pack_bf16(x[6], x[7]);
            *reinterpret_cast<uint4*>(a.out.data + row * a.out.stride_row + head * a.out.stride_head + c0 + col) = v;
            if (a.lse != nullptr && c0 + col == 0) a.lse[row * a.lse_stride_row + head * a.lse_stride_head] = row_lse(all);
          } else {
            float4* dst = reinterpret_cast<float4*>(args.parts.sums + ((int64_t)slot * R + r) * D + c0 + col);
            dst[0] = make_float4(x[0], x[1], x[2], x[3]);
            dst[1] = make_float4(x[4], x[5], x[6], x[7]);
            if (c0 + col == 0) args.parts.stats[slot * R + r] = make_float4(all.m, all.m_sum, all.l, 0.f);
          }
        }
        if (!join.wait(ab)) return;
      }
      if ((flags & kFromStart) && !(flags & kToEnd) && threadIdx.x == 0) {
        args.parts.headers[2 * blockIdx.x] = make_int4(flags >> 8, d.row0, d.head, d.row_tile);
        args.parts.headers[2 * blockIdx.x + 1] = make_int4(live, 0, 0, 0);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the stage was written with ordinary stores; copies follow
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.empty[stage]));
    if (++stage == T::STAGES) stage = 0, parity ^= 1;
  }
}

template <int D, int BITS, int R>
__global__ void __launch_bounds__(Traits<D, BITS, R>::THREADS, Traits<D, BITS, R>::CTAS) attend_step_kernel(const __grid_constant__ StepArgs args) {
  using T = Traits<D, BITS, R>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring_ptr = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  unsigned char* q_tile = ring_ptr + T::STAGES * T::STAGE;
  SmallSmem& sm = *reinterpret_cast<SmallSmem*>(q_tile + T::QBYTES);
  if (threadIdx.x == 0) {
    for (int i = 0; i < T::STAGES; ++i) {
      mbar_init(smem_u32(&sm.full[i]), 1);
      mbar_init(smem_u32(&sm.empty[i]), kWarps);
    }
    mbar_init(smem_u32(&sm.join), kWarps);
    sm.abort = 0;
    args.parts.headers[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  find_start<T>(args, sm);                               // ends with a barrier of the CTA
  grid_launch_dependents();                              // every CTA of this kernel has started: the joining one can take its place
  const int64_t total = sm.total;
  const int64_t per = (total + gridDim.x - 1) / gridDim.x;
  const int64_t w0 = per * blockIdx.x, w1 = min(w0 + per, total);
  if (w0 < w1) {
    const Abort ab{&sm.abort, args.a.dev_status};
    if (threadIdx.x < kWarps * 32) {
      if constexpr (T::LEND) reg_inc<kComputeRegs>();
      compute_tiles<T>(args, sm, ring_ptr, smem_u32(ring_ptr), q_tile, w0, w1 - w0, ab);
    } else {
      if constexpr (T::LEND) reg_dec<kOtherRegs>();
      if (threadIdx.x < (kWarps + 1) * 32) copy_tiles<T>(args, sm, smem_u32(ring_ptr), w0, w1, per, ab);
    }
  }
}

// Rows of a tile: the fewest that hold the rows of a sequence and key head.
int tile_rows(const spf_kv_cache* cache, int group, int max_new) {
  const int64_t rows = (int64_t)group * max_new;
  return rows <= 8 ? 8 : rows <= 16 ? 16 : step_rows(cache);
}
int ctas_per_sm(int rows) { return rows <= 8 ? 3 : 2; }

template <int D, int BITS, int R>
int32_t launch_step(StepArgs& args, const spf_kv_cache* cache, int live, int ctas, cudaStream_t stream) {
  using T = Traits<D, BITS, R>;
  static ContextSet done;
  int32_t st = encode_pool_map("spf_attend", cache, cache->k_pool, T::KEYS, &args.k_map);
  if (st == SPF_OK) st = encode_pool_map("spf_attend", cache, cache->v_pool, T::KEYS, &args.v_map);
  if constexpr (T::INT4) {
    if (st == SPF_OK) st = encode_scale_map("spf_attend", cache, cache->k_scale, &args.k_scale_map);
    if (st == SPF_OK) st = encode_scale_map("spf_attend", cache, cache->v_scale, &args.v_scale_map);
  }
  if (st == SPF_OK) st = allow_shared_memory(reinterpret_cast<const void*>(attend_step_kernel<D, BITS, R>), smem_bytes<T>(), done);
  if (st != SPF_OK) return st;
  attend_step_kernel<D, BITS, R><<<ctas, T::THREADS, smem_bytes<T>(), stream>>>(args);
  SPF_CUDA_CHECK(cudaGetLastError());
  return attend_join_launch(args.a, args.parts, R, live, D, T::FP8, ctas, stream);
}

template <int D, int BITS>
int32_t launch_rows(StepArgs& args, const spf_kv_cache* cache, int rows, int live, int ctas, cudaStream_t stream) {
  switch (rows) {
    case 8: return launch_step<D, BITS, 8>(args, cache, live, ctas, stream);
    case 16: break;
    default:
      if constexpr (D == 64 || BITS == 16) return launch_step<D, BITS, 32>(args, cache, live, ctas, stream);
  }
  return launch_step<D, BITS, 16>(args, cache, live, ctas, stream);
}

}  // namespace

size_t attend_step_workspace_bytes(const spf_kv_cache* cache, int group, int max_new, int sm_count) {
  // a step with fewer rows has more CTAs: the most that any with up to this many takes
  size_t most = 0;
  for (int rows = 8; rows <= tile_rows(cache, group, max_new); rows *= 2)
    most = std::max(most, parts_layout(rows, cache->head_dim, sm_count * ctas_per_sm(rows)).total);
  return most;
}

int32_t attend_step_launch(const AttendArgs& a, const spf_kv_cache* cache, int max_new, int sm_count, void* workspace, cudaStream_t stream) {
  StepArgs args{};
  args.a = a;
  const int rows = tile_rows(cache, a.group, max_new), live = (int)std::min<int64_t>((int64_t)a.group * max_new, rows), ctas = sm_count * ctas_per_sm(rows);
  args.parts = parts_at(workspace, rows, cache->head_dim, ctas);
  const bool d64 = cache->head_dim == 64;
  switch (a.kv.bits) {
    case 4: return d64 ? launch_rows<64, 4>(args, cache, rows, live, ctas, stream) : launch_rows<128, 4>(args, cache, rows, live, ctas, stream);
    case 8: return d64 ? launch_rows<64, 8>(args, cache, rows, live, ctas, stream) : launch_rows<128, 8>(args, cache, rows, live, ctas, stream);
    default: return d64 ? launch_rows<64, 16>(args, cache, rows, live, ctas, stream) : launch_rows<128, 16>(args, cache, rows, live, ctas, stream);
  }
}

}  // namespace spf
