// Attention with few rows per key head: what the kernels that read a cache's tiles for a step's rows share (the attention, the weights that
// keys receive).  Warp-level products with keys as the 16 rows of the left operand and query rows as the 8 columns of the right one.
#pragma once

#include "attend.cuh"

namespace spf {
namespace {

constexpr int kWarps = 4;               // that compute
// A second warpgroup, whose first warp copies, lends registers of the 128 a thread that the launch has: 128 x (192 + 64) = 256 x 128.
constexpr int kComputeRegs = 192, kOtherRegs = 64;
constexpr int kMaxStages = 8;


// What the copying warp tells the computing ones about a stage.
struct TileDesc {
  int row0, n_new, pos0, first, end, head, row_tile, key0;
  float k_scale[2], v_log2[2];          // 8 bits: of the tile's groups of 64 keys
  int flags;                            // kFirst, kLast, kNoKeys; bits 8 ...: CTAs behind this one with parts of the triple
};


template <int D_, int BITS_, int R_, bool VALUES_ = true>
struct Traits {
  static constexpr int D = D_, BITS = BITS_, R = R_;
  static constexpr bool FP8 = BITS == 8, INT4 = BITS == 4, VALUES = VALUES_;   // VALUES: the tiles have values beside the keys
  // Warps over rows and over keys: a warp's outputs are 32 registers (8 rows of 128 dimensions, 16 of 64).  With 64 of them, 32 rows
  // of 64 dimensions took 69 instead of 61 us (131072 keys, 8 heads), though each key is then read by half as many warps.
  static constexpr int WR = !VALUES || R * D <= 1024 ? 1 : R * D / 1024, WK = kWarps / WR;
  static constexpr int NT = R / (8 * WR);                             // 8-row tiles of a warp
  // Keys of a tile: 128 where their rows are short, so that a warp has two sixteens of them at a time.  (One sixteen is a chain of
  // dependent steps: with tiles of 64 keys 32 sequences of up to 16k tokens on an 8-bit cache took 136 instead of 111 us, four of up to
  // 250k 384 instead of 292, eight lookahead tokens over 131072 keys of 64 dimensions 92 instead of 70.)  A warp's keys share a scale, so they are 64 at most; 4 bits: they do not.
  static constexpr int KEYS = INT4 || ((FP8 ? D : 2 * D) <= 128 && WK > 1) ? 128 : 64;
  static constexpr int KW = KEYS / WK, KT = KW / 16;                  // keys of a warp in a tile, in sixteens
  static constexpr bool LEND = VALUES && R >= 16 && R * D < 4096;     // registers move between warpgroups
  static constexpr int THREADS = LEND ? 2 * kWarps * 32 : (kWarps + 1) * 32;
  // Per SM.  Without values, whose sums are not there: 8 rows 61 us with four, 71 with three (a token of 32 sequences, 4 bits); 128 rows 92 with
  // three, 104 with two (131072 keys of 64 dimensions, bf16).
  static constexpr int CTAS = R == 8 ? (VALUES ? 3 : 4) : VALUES ? 2 : 3;
  static constexpr int WTERMS = BITS == 16 && R == 8 ? 2 : 1;               // of a weight
  static constexpr bool QREGS = NT <= 2 && !(VALUES && INT4 && R * D == 1024);   // queries stay in registers, where there is room (4 bits, 128 dimensions: 77 us without, 85 with them)
  static constexpr int ROWB = D * BITS / 8, SPAN = ROWB < 128 ? ROWB : 128;
  // A stage: the keys, the values; 4 bits: their scales behind them.
  static constexpr int PARTS = D / kScaleDims, TILE = KEYS * ROWB, SCALES = INT4 ? KEYS * PARTS * 2 : 0, STAGE = (VALUES ? 2 : 1) * (TILE + SCALES);
  // 8-bit keys are multiplied as they are, by queries in two 8-bit terms, where their logits make an attention; where weights are an output
  // of their own (no values), in bf16: sums of 8-bit products are cut off earlier and left 1.3e-6 in them, also with a third term, and
  // bf16 ones 6e-8.
  static constexpr bool WIDE = FP8 && !VALUES;
  static constexpr int TERMS = FP8 && !WIDE ? 2 : 1;
  static constexpr int QBYTES = R * D * 2;
  // Row tiles whose queries are kept: without values, where nothing is left behind for a row, keys wait for all of them.
  static constexpr int TILES_HELD = !VALUES && R == 32 ? 4 : 1;
  static constexpr int FIT = ((CTAS == 4 ? 55 : CTAS == 3 ? 74 : 112) * 1024 - 4096 - TILES_HELD * QBYTES) / STAGE;
  static constexpr int STAGES = FIT < kMaxStages ? FIT : kMaxStages;
  static constexpr int JOIN = D * WK * R * 4 <= 2 * TILE ? D : 2 * TILE / (WK * R * 4);   // output columns joined at a time
};

enum : int { kFirst = 1, kLast = 2, kNoKeys = 4, kFromStart = 8, kToEnd = 16 };

struct SmallSmem {
  unsigned long long full[kMaxStages], empty[kMaxStages], join;
  TileDesc desc[kMaxStages];
  RowStats stats[kWarps][32];           // of the warps' rows
  int64_t scan[2 * kWarps];
  int64_t total, start_base;
  int start_seq;
  int abort;
};

template <class T>
constexpr int smem_bytes() { return T::STAGES * T::STAGE + T::QBYTES + (int)sizeof(SmallSmem) + 1024; }

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

template <bool FP8>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (FP8)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The same onto other sums, bf16.
__device__ __forceinline__ void mma16_from(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// 8-bit keys by the E4M3 (LOW: E5M2) term of 8-bit queries.
template <bool LOW>
__device__ __forceinline__ void mma32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (LOW)
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e5m2.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of the 16-byte chunk `chunk` of row `row` in a tile, as the copies' swizzle lays it: spans of 128 (or 64) bytes
// one after the other, the chunk's place in its span exchanged by the row.
template <class T>
__device__ __forceinline__ uint32_t tile_chunk(int row, int chunk) {
  if constexpr (T::SPAN == 32) return (uint32_t)(row * 32 + ((chunk ^ (row >> 2)) & 1) * 16);
  if constexpr (T::SPAN == 64) return (uint32_t)(row * 64 + ((chunk ^ (row >> 1)) & 3) * 16);
  return (uint32_t)((chunk >> 3) * (T::KEYS * 128) + row * 128 + ((chunk ^ row) & 7) * 16);
}
// The same for the query tile, rows of 2 D bytes.
template <class T>
__device__ __forceinline__ uint32_t q_chunk(int row, int chunk) {
  return (uint32_t)(row * (2 * T::D) + ((chunk & ~7) | ((chunk ^ row) & 7)) * 16);
}

// One term of 8-bit queries, rows of D bytes: eight rows' chunks of one column on banks of their own.
template <class T>
__device__ __forceinline__ uint32_t q8_chunk(int row, int chunk) {
  if constexpr (T::D == 64) return (uint32_t)(row * 64 + ((chunk ^ (row >> 1)) & 3) * 16);
  return (uint32_t)(row * 128 + ((chunk ^ row) & 7) * 16);
}

// ---------------------------------------------------------------------------------------------- queries and keys
// 4 bits: the exponent e by which a row of queries is scaled, 2^e taking its largest element to about 2^120.  It is clipped where 2^e would
// leave fp32's range, or the factor 2^(133 - e) to logits would.
__device__ __forceinline__ int code_exponent(float top) { return min(max(247 - (int)(__float_as_uint(top) >> 23), 6), 120); }

// What a row's logits need besides its elements.
template <class T>
struct QueryNotes {
  float factor[T::R];                                    // 8 bits: 2^-e (in bf16: 2^(120 - e)); 4 bits: c 2^(133 - e)
  float base[T::INT4 ? T::PARTS : 1][T::R];              // 4 bits: -8 2^-133 times the sum of 32 scaled elements
};

// The triple's query rows into shared memory, rows that do not exist as zeros (without values, whose weights are added up over rows: as the last
// one).  8 bits: the two terms, one tile behind the other.  4
// bits: scaled by 2^e, eight elements in the order 0 4 2 6 1 5 3 7 in which codes come out of a word, the latter four by 1/16 of that; 8 bits in
// bf16: scaled too, four elements in the order 0 2 1 3 in which bytes do.
template <class T>
__device__ __forceinline__ void load_queries(const AttendArgs& a, const TileDesc& d, unsigned char* q_tile, QueryNotes<T>& notes) {
  constexpr int kLanes = T::D / 8;                       // threads of a row
  const int total = d.n_new * a.group;
  for (int item = threadIdx.x; item < T::R * kLanes; item += kWarps * 32) {
    const int r = item / kLanes, part = item % kLanes, rr = T::VALUES ? d.row_tile * T::R + r : min(d.row_tile * T::R + r, total - 1);
    const __nv_bfloat16* src = a.q.data + (int64_t)(d.row0 + rr / a.group) * a.q.stride_row + (int64_t)(d.head * a.group + rr % a.group) * a.q.stride_head;
    union { uint4 u; __nv_bfloat162 h[4]; } v;
    v.u = make_uint4(0, 0, 0, 0);
    if (rr < total) v.u = __ldg(reinterpret_cast<const uint4*>(src) + part);
    if constexpr (T::BITS == 16) {
      *reinterpret_cast<uint4*>(q_tile + q_chunk<T>(r, part)) = v.u;
    } else {
      float f[8];
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 p = __bfloat1622float2(v.h[i]);
        f[2 * i] = p.x, f[2 * i + 1] = p.y;
        top = fmaxf(top, fmaxf(fabsf(p.x), fabsf(p.y)));
      }
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o, kLanes));
      if constexpr (T::TERMS == 2) {
        int e;
        uint2 hi, lo;
        two_terms(f, top, &e, &hi, &lo);
        *reinterpret_cast<uint2*>(q_tile + q8_chunk<T>(r, part >> 1) + 8 * (part & 1)) = hi;
        *reinterpret_cast<uint2*>(q_tile + T::R * T::D + q8_chunk<T>(r, part >> 1) + 8 * (part & 1)) = lo;
        if (part == 0) notes.factor[r] = __uint_as_float((uint32_t)(127 - e) << 23);
      } else {
        const int e = code_exponent(top);
        const float up = __uint_as_float(top == INFINITY ? 0x7fffffffu : (uint32_t)(e + 127) << 23), up16 = up * 0.0625f;
        if constexpr (T::WIDE) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int o = 8 * (part & 3) + 4 * i;        // of the 32 dimensions: lane (o % 16) / 4 has four of either 16
            *reinterpret_cast<uint2*>(q_tile + q_chunk<T>(r, (part & ~3) + ((o & 15) >> 2)) + 8 * (o >> 4)) =
                make_uint2(pack_bf16(f[4 * i] * up, f[4 * i + 2] * up), pack_bf16(f[4 * i + 1] * up, f[4 * i + 3] * up));
          }
          if (part == 0) notes.factor[r] = __uint_as_float((uint32_t)(120 - e + 127) << 23);
          continue;
        }
        *reinterpret_cast<uint4*>(q_tile + q_chunk<T>(r, part)) = make_uint4(pack_bf16(f[0] * up, f[4] * up), pack_bf16(f[2] * up, f[6] * up),
                                                                           pack_bf16(f[1] * up16, f[5] * up16), pack_bf16(f[3] * up16, f[7] * up16));
        float sum = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if ((part & 3) == 0) notes.base[part >> 2][r] = sum * -__uint_as_float((uint32_t)(e - 130 + 127) << 23);
        if (part == 0) notes.factor[r] = fminf(a.c * __uint_as_float((uint32_t)(133 - e + 127) << 23), 3.402823466e38f);
      }
    }
  }
}

// The queries of 8 rows as right operands for 32 (8 bits: 64) dimensions: b[0..1] of two products; 8 bits: first[0..1], second[2..3]
// of one term.
template <class T>
__device__ __forceinline__ void query_operand(uint32_t q_addr, int row, int step, int lane, uint32_t (&b)[4]) {
  if constexpr (T::INT4 || T::WIDE) {
    // four lanes have 32 elements, eight each, one behind the other
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3])
                 : "r"(q_addr + q_chunk<T>(row + (lane >> 2), 4 * step + (lane & 3))));
  } else if constexpr (T::FP8) ldsm4(q_addr + q8_chunk<T>(row + (lane & 7), 4 * step + (lane >> 3)), b);
  else ldsm4(q_addr + q_chunk<T>(row + (lane & 7), 4 * step + (lane >> 3)), b);
}

// The key (of sixteen) in row r of the first (half = 0) or second eight rows of a left operand.  8 bits: the even and the odd keys, as the
// values' bytes come.  4 bits: 0-3 and 12-15, 4-11: a copy of eight 16-byte pieces for the keys' operand then touches every bank once, and
// so does one for the values', whose rows are those of both halves in turns.
template <class T>
__device__ __forceinline__ int operand_key(int r, int half) {
  if constexpr (T::INT4) return half ? r + 4 : r + 2 * (r & 4);
  return T::FP8 && T::VALUES ? 2 * r + half : r + 8 * half;
}
// The 16 keys from `key` on as the left operand: bf16 16 dimensions (of chunk pair `step`), 8 bits 32; 4 bits: words of eight codes of two
// times 32 dimensions.
template <class T>
__device__ __forceinline__ void key_operand(uint32_t k_tile, int key, int step, int lane, uint32_t (&a)[4]) {
  ldsm4(k_tile + tile_chunk<T>(key + operand_key<T>(lane & 7, (lane >> 3) & 1), 2 * step + (lane >> 4)), a);
}
// The key (from the warp's sixteen) of a thread's logits 0, 1 (half = 0) and 2, 3 (half = 1).
template <class T>
__device__ __forceinline__ int key_of(int lane, int half) { return operand_key<T>(lane >> 2, half); }

// What a thread keeps of a triple's queries.
template <class T>
struct Queries {
  static constexpr int kTerms = T::TERMS, kSteps = kTerms == 2 ? T::D / 64 : T::D / 32;   // four registers each
  uint32_t q[T::QREGS ? kTerms * kSteps * T::NT : 1][4];
  float factor[T::NT][2];                                // of its rows, 2 (lane % 4) and the next of every 8
  float base[T::INT4 ? T::PARTS : 1][T::INT4 ? T::NT : 1][2];

  __device__ __forceinline__ void load(uint32_t q_addr, const QueryNotes<T>& notes, int row_off, int lane) {
#pragma unroll
    for (int nt = 0; nt < T::NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = row_off + nt * 8 + 2 * (lane & 3) + e;
        if constexpr (T::BITS != 16) factor[nt][e] = notes.factor[row];
        if constexpr (T::INT4) {
#pragma unroll
          for (int p = 0; p < T::PARTS; ++p) base[p][nt][e] = notes.base[p][row];
        }
      }
    if constexpr (T::QREGS) {
#pragma unroll
      for (int t = 0; t < kTerms; ++t)
#pragma unroll
        for (int x = 0; x < kSteps; ++x)
#pragma unroll
          for (int nt = 0; nt < T::NT; ++nt) query_operand<T>(q_addr + t * T::R * T::D, row_off + nt * 8, x, lane, q[(t * kSteps + x) * T::NT + nt]);
    }
  }
  __device__ __forceinline__ void operand(uint32_t q_addr, int row_off, int t, int x, int nt, int lane, uint32_t (&b)[4]) const {
    if constexpr (T::QREGS) {
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = q[(t * kSteps + x) * T::NT + nt][e];
    } else {
      query_operand<T>(q_addr + t * T::R * T::D, row_off + nt * 8, x, lane, b);
    }
  }
};

// The scales of a key's (value's) elements, 4 bits.
template <class T>
__device__ __forceinline__ void load_scales(uint32_t scales, int key, float (&s)[T::PARTS]) {
  uint32_t w[T::PARTS / 2];
  if constexpr (T::PARTS == 4) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(scales + key * 8));
  else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(scales + key * 4));
#pragma unroll
  for (int p = 0; p < T::PARTS; ++p) s[p] = __uint_as_float(p & 1 ? w[p / 2] & 0xffff0000u : w[p / 2] << 16);
}

// Products of the warp's keys (of the tile, from `key` on) and rows; base-2 logits are these times a factor.
//
// 4 bits: codes are multiplied as they are, without being converted: a code in the low (or in the second) four bits of a half is the
// subnormal bf16 number code 2^-133 (16 times that), and one instruction makes two of them of a word.  The products of 32 dimensions, which
// share a scale, start from -8 times the sum of their query elements.  Queries are scaled by 2^e, which takes a row's largest to 2^120, so
// that sums stay in fp32's normal range.
template <class T>
__device__ __forceinline__ void tile_logits(float (&z)[T::KT][T::NT][4], const Queries<T>& queries, uint32_t q_addr, int row_off, uint32_t k_tile, uint32_t scales,
                                            int key, int lane) {
  constexpr int NT = T::NT, KT = T::KT, kTerms = Queries<T>::kTerms, kSteps = Queries<T>::kSteps;
  if constexpr (T::INT4) {
    float s[KT][2][T::PARTS];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int h = 0; h < 2; ++h) load_scales<T>(scales, key + kt * 16 + key_of<T>(lane, h), s[kt][h]);
#pragma unroll
    for (int x = 0; x < T::PARTS / 2; ++x) {
      uint32_t w[KT][4];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) key_operand<T>(k_tile, key + kt * 16, x, lane, w[kt]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int p = 2 * x + h;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          uint32_t b[4];
          queries.operand(q_addr, row_off, 0, p, nt, lane, b);
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            const uint32_t lo = w[kt][2 * h], hi = w[kt][2 * h + 1];
            const uint32_t first[4] = {lo & 0x000f000fu, hi & 0x000f000fu, (lo >> 8) & 0x000f000fu, (hi >> 8) & 0x000f000fu},
                           second[4] = {lo & 0x00f000f0u, hi & 0x00f000f0u, (lo >> 8) & 0x00f000f0u, (hi >> 8) & 0x00f000f0u};
            const float base[4] = {queries.base[p][nt][0], queries.base[p][nt][1], queries.base[p][nt][0], queries.base[p][nt][1]};
            float acc[4];
            mma16_from(acc, first, b[0], b[1], base);
            mma16<false>(acc, second, b[2], b[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[kt][nt][e] = p == 0 ? s[kt][e >> 1][p] * acc[e] : fmaf(s[kt][e >> 1][p], acc[e], z[kt][nt][e]);
          }
        }
      }
    }
  } else if constexpr (T::WIDE) {
    // A byte s eeee mmm moved to the bits s 0000eeee mmm0000 of a bf16 number is its value times 2^-120, subnormals included.  The NaN patterns
    // look like 480 then, so they are looked for.
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[kt][nt][e] = 0.f;
    uint32_t nan[KT][2] = {};
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {
      uint32_t w[KT][4];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        key_operand<T>(k_tile, key + kt * 16, x, lane, w[kt]);
#pragma unroll
        for (int i = 0; i < 4; ++i) nan[kt][i & 1] |= (w[kt][i] & 0x7f7f7f7fu) + 0x01010101u;
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        uint32_t b[4];
        queries.operand(q_addr, row_off, 0, x, nt, lane, b);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t lo = w[kt][2 * h], hi = w[kt][2 * h + 1];
            const uint32_t a[4] = {((lo << 8) & 0x80008000u) | ((lo << 4) & 0x07f007f0u), ((hi << 8) & 0x80008000u) | ((hi << 4) & 0x07f007f0u),
                                   (lo & 0x80008000u) | ((lo >> 4) & 0x07f007f0u), (hi & 0x80008000u) | ((hi >> 4) & 0x07f007f0u)};
            mma16<false>(z[kt][nt], a, b[2 * h], b[2 * h + 1]);
          }
      }
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!__any_sync(0xffffffffu, (nan[kt][h] & 0x80808080u) != 0)) continue;
        const uint32_t row = 0xfu << (lane & 28);        // the four lanes of a key
        if ((__ballot_sync(0xffffffffu, (nan[kt][h] & 0x80808080u) != 0) & row) == 0) continue;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) z[kt][nt][2 * h] = z[kt][nt][2 * h + 1] = __uint_as_float(0x7fffffffu);
      }
  } else {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[kt][nt][e] = 0.f;
#pragma unroll
    for (int x = 0; x < kSteps; ++x) {
      uint32_t k[KT][2][4];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int h = 0; h < 2; ++h) key_operand<T>(k_tile, key + kt * 16, 2 * x + h, lane, k[kt][h]);
#pragma unroll
      for (int t = 0; t < kTerms; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          uint32_t b[4];
          queries.operand(q_addr, row_off, t, x, nt, lane, b);
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if constexpr (!T::FP8) mma16<false>(z[kt][nt], k[kt][h], b[2 * h], b[2 * h + 1]);
              else if (t == 0) mma32<false>(z[kt][nt], k[kt][h], b[2 * h], b[2 * h + 1]);
              else mma32<true>(z[kt][nt], k[kt][h], b[2 * h], b[2 * h + 1]);
            }
        }
    }
  }
}

}  // namespace
}  // namespace spf
