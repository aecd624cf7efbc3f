// Rotation of a step's queries and keys by position, and the append of keys and values to the paged cache.
//
//   q'[t, h] = R(p_t) q[t, h],  k'[t, h] = R(p_t) k[t, h],  R(p): pairs (x, y) -> (x cos - y sin, y cos + x sin), fp32, each
//   product rounded by itself (no fused multiply-add: the result is then the same wherever the formula is written out).
//
// bf16 pools: one rounding, straight to the token's place.  8-bit pools: a scale belongs to 64 tokens of a block and head, so
// one CTA makes the new tokens of such a group, their largest magnitude, the scale, and the bytes:
//   s' = max(s of the tokens that the group holds already, 2^ceil(log2(max |x| / 448))),   byte = E4M3(x / s'),
// and rounds the bytes held already from s to s' where it grew.  Powers of two: that second rounding is then exact but for
// bytes that become subnormal.  4-bit pools: a token's 32 consecutive elements of a head have a scale of their own,
//   s = the smallest number of five significant bits with 7 s >= max |x|,   code = 8 + rint(x (1 / s)),
// so that tokens are independent, as with bf16, and a row is moved by the same threads: the D / 16 lanes that have a head's elements
// exchange their largest magnitudes, and each writes the codes of its two runs of 8, 4 bytes each.
//
// Bounds: bytes for a prompt, a launch and four dependent loads (row_start, seq_lens, table, the data) for single tokens.
#include <algorithm>
#include <type_traits>

#include <cuda_fp16.h>

#include "kv.cuh"
#include "tc_ptx.cuh"

namespace spf {
namespace {

constexpr int kAppendThreads = 256;

struct AppendArgs {
  KvView kv;
  StepView step;
  RowsView k, v, q, q_out;
  const float* rope;            // null: no rotation
  const int32_t* positions;     // null: a token's place in its sequence
  int n_positions, rot_dim, interleaved;
  int n_q_heads;                // 0: no queries in this call
  int rotate_ctas;              // CTAs that move whole rows; before them, those that fill 8-bit groups
  int fill_heads;               // heads whose keys and values such a CTA fills (where there are many)
  uint64_t per_row_inverse;     // 2^64 / (threads of a row), rounded up
  int32_t* dev_status;
};

union Pack8 {
  uint4 u;
  __nv_bfloat162 h[4];
};

__device__ __forceinline__ uint4 load_raw(const __nv_bfloat16* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

__device__ __forceinline__ void widen8(const uint4& raw, float (&x)[8]) {
  Pack8 v;
  v.u = raw;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __bfloat1622float2(v.h[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

__device__ __forceinline__ uint4 narrow8(const float (&x)[8]) {
  Pack8 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v.h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
  return v.u;
}

// A head is moved in units of 16 elements, two runs of 8: where the unit's halves lie, and which angles turn them (angle < 0:
// the unit is not rotated).  Units of the split form pair element j with j + rot_dim / 2.
struct Unit {
  int first, second, angle;
};
__device__ __forceinline__ Unit unit_of(int u, int rot_dim, int interleaved) {
  if (u * 16 >= rot_dim) return Unit{u * 16, u * 16 + 8, -1};
  if (interleaved) return Unit{u * 16, u * 16 + 8, u * 8};
  return Unit{u * 8, rot_dim / 2 + u * 8, u * 8};
}

// Cosines and sines of four of a unit's eight pairs, the first four or the others.
struct Angles {
  float4 c, s;
};
__device__ __forceinline__ Angles load_angles(const float* table, int64_t row, int rot_dim, int angle) {
  const float* at = table + row * rot_dim + angle;
  return Angles{__ldg(reinterpret_cast<const float4*>(at)), __ldg(reinterpret_cast<const float4*>(at + rot_dim / 2))};
}

__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// (Packed pairs, mul.rn.f32x2 and add.rn.f32x2, gave other last bits: the two were made one instruction.)
__device__ __forceinline__ void turn(float& x, float& y, float c, float s) {
  const float nx = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
  y = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
  x = nx;
}
__device__ __forceinline__ void rotate(float (&a)[8], float (&b)[8], const Angles& t, int half, int interleaved) {
  const float c[4] = {t.c.x, t.c.y, t.c.z, t.c.w}, s[4] = {t.s.x, t.s.y, t.s.z, t.s.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!interleaved) turn(a[4 * half + i], b[4 * half + i], c[i], s[i]);
    else if (half == 0) turn(a[2 * i], a[2 * i + 1], c[i], s[i]);
    else turn(b[2 * i], b[2 * i + 1], c[i], s[i]);
  }
}

// Position in the sequence and row of the angles' table; false (and reported) where one lies outside.
__device__ __forceinline__ bool place_of(const AppendArgs& a, int seq, int row, int* pos, int64_t* angle_row) {
  const int start = __ldg(a.step.row_start + seq), end = __ldg(a.step.row_start + seq + 1), len = __ldg(a.step.seq_lens + seq);
  *pos = place_from_end(len, (int64_t)end - row);
  *angle_row = a.positions != nullptr ? __ldg(a.positions + row) : *pos;
  const bool fine = row >= start && *pos >= 0 && (a.rope == nullptr || (*angle_row >= 0 && *angle_row < a.n_positions));
  if (!fine) report_cache(a.dev_status);
  return fine;
}

// ---------------------------------------------------------------------------------------------- 4-bit rows
// Largest magnitude of eight elements, as bits that order like it: infinities as zeros, NaN above every number.
__device__ __forceinline__ uint32_t largest_bits(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  if (top == 0x7f800000u) {
    top = 0;                                        // some are infinite, none is NaN: once more without them
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t m = __float_as_uint(x[i]) & 0x7fffffffu;
      top = max(top, m == 0x7f800000u ? 0u : m);
    }
  }
  return top;
}
// The smallest number of five significant bits s >= 2^-100 with 7 s >= the magnitude; NaN for NaN.
__device__ __forceinline__ float short_scale(uint32_t magnitude) {
  if (magnitude > 0x7f800000u) return __uint_as_float(0x7fc00000u);
  // a seventh but for a rounding, cut to five bits, is that number or the one below it, and 7 times either is exact (3 + 5 bits)
  const float top = __uint_as_float(magnitude);
  uint32_t s = __float_as_uint(top * (1.f / 7.f)) & 0xfff80000u;
  if (__uint_as_float(s) * 7.f < top) s += 0x80000u;
  return fmaxf(__uint_as_float(s), 0x1p-100f);
}
// Codes of eight elements, the first in the lowest four bits.
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], float inverse) {
  uint32_t two[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t c[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float t = fminf(fmaxf(__fmul_rn(x[2 * i + e], inverse), -7.f), 7.f);
      c[e] = __float_as_uint(__fadd_rn(t, 12582920.f));   // 1.5 * 2^23 + 8: the sum's last byte is the code
    }
    two[i] = c[0] + 16u * c[1];
  }
  return __byte_perm(__byte_perm(two[0], two[1], 0x0040), __byte_perm(two[2], two[3], 0x0040), 0x5410);
}
// A head's row of a 4-bit pool: its D / 16 lanes, neighbours in a warp, have a unit each.  `whole`: units are those of a head that is
// rotated as a whole, in the split form (1), or two runs side by side (2); else (0) they may be either.
template <int D>
__device__ __forceinline__ void write_codes(uint8_t* row, uint16_t* scales, const float (&f)[8], const float (&g)[8], const Unit& u, int whole) {
  constexpr int kUnits = D / 16, kParts = D / kScaleDims;
  const uint32_t lanes = ((1u << kUnits) - 1u) << (threadIdx.x & 31 & ~(kUnits - 1));
  uint32_t mf = largest_bits(f), mg = largest_bits(g);
  if (whole == 1) {
    // four neighbours have the first, and the second, runs of 32 elements each
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      mf = max(mf, __shfl_xor_sync(lanes, mf, o));
      mg = max(mg, __shfl_xor_sync(lanes, mg, o));
    }
  } else if (whole == 2) {
    mf = max(mf, mg);                               // two neighbours have 32 elements
    mf = mg = max(mf, __shfl_xor_sync(lanes, mf, 1));
  } else {
    uint32_t of_f = 0, of_g = 0;
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
      uint32_t m = max(u.first / kScaleDims == p ? mf : 0u, u.second / kScaleDims == p ? mg : 0u);
#pragma unroll
      for (int o = 1; o < kUnits; o <<= 1) m = max(m, __shfl_xor_sync(lanes, m, o));
      if (u.first / kScaleDims == p) of_f = m;
      if (u.second / kScaleDims == p) of_g = m;
    }
    mf = of_f, mg = of_g;
  }
  const float sf = short_scale(mf), sg = whole == 2 ? sf : short_scale(mg), inverse = __frcp_rn(sf);
  *reinterpret_cast<uint32_t*>(row + u.first / 2) = codes8(f, inverse);
  *reinterpret_cast<uint32_t*>(row + u.second / 2) = codes8(g, whole == 2 ? inverse : __frcp_rn(sg));
  // who has the first run of 32 elements writes their scale
  if (u.first % kScaleDims == 0) scales[u.first / kScaleDims] = (uint16_t)(__float_as_uint(sf) >> 16);
  if (u.second % kScaleDims == 0) scales[u.second / kScaleDims] = (uint16_t)(__float_as_uint(sg) >> 16);
}

// Rows one by one: queries (always), keys and values (bf16 and 4-bit pools).  A thread has one unit of HPT heads of a row, so that a
// row's angles are read once for HPT heads.
template <int D, int HPT, int BITS>
__device__ __forceinline__ void move_rows(const AppendArgs& a, int cta) {
  constexpr int kUnits = D / 16;
  const int turned = a.n_q_heads + (BITS == 8 ? 0 : a.kv.n_kv_heads), copied = BITS == 8 ? 0 : a.kv.n_kv_heads;
  const int turned_groups = (turned + HPT - 1) / HPT, groups = turned_groups + (copied + HPT - 1) / HPT;
  const int per_row = groups * kUnits;
  const int64_t first = (int64_t)cta * kAppendThreads, item = first + threadIdx.x;
  // n / per_row = high word of n ceil(2^64 / per_row) while n per_row < 2^64 (here below 2^39 and 2^20): a 64-bit division by a
  // value that is not known when this is compiled takes some hundred instructions, more than everything else here
  auto row_of = [&](int64_t n) { return (int)__umul64hi((uint64_t)n, a.per_row_inverse); };
  // the sequences of the CTA's first and last row, by one look of all threads at the starts; a thread's own lies between
  const int row_lo = row_of(first), row_hi = min(row_of(first + kAppendThreads - 1), a.step.n_rows - 1);
  int lo = 0, hi = 0;
  for (int b = 0; b < a.step.n_seqs; b += kAppendThreads) {
    const int start = b + (int)threadIdx.x < a.step.n_seqs ? __ldg(a.step.row_start + b + threadIdx.x) : 0x7fffffff;
    lo += __syncthreads_count(start <= row_lo);
    hi += __syncthreads_count(start <= row_hi);
  }
  const int row = row_of(item);
  if (row >= a.step.n_rows || row >= __ldg(a.step.row_start + a.step.n_seqs)) return;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(a.step.row_start + mid) <= row) lo = mid + 1;
    else hi = mid;
  }
  const int seq = lo - 1;
  if (seq < 0) return;
  int pos;
  int64_t angle_row;
  if (!place_of(a, seq, row, &pos, &angle_row)) return;
  const int in_row = (int)(item - (int64_t)row * per_row), group = in_row / kUnits;
  const Unit u = unit_of(in_row % kUnits, a.rope != nullptr ? a.rot_dim : 0, a.interleaved);
  const bool copy = group >= turned_groups;
  const int whole = a.rope == nullptr ? 2 : a.rot_dim < D ? 0 : a.interleaved ? 2 : 1;   // 4 bits
  const int head0 = (copy ? group - turned_groups : group) * HPT, heads = copy ? copied : turned;

  const int64_t block = pool_block(a.kv, a.step, seq, pos);
  if (block < 0) {
    report_cache(a.dev_status);
    return;
  }
  // the token's row in a pool, but for the head
  const int64_t cell = block * a.kv.n_kv_heads * a.kv.block_tokens + pos % a.kv.block_tokens;
  const bool turns = !copy && u.angle >= 0;
  uint4 x[HPT][2];                                  // what is not turned is copied as it is
  Angles t[2];
  if (turns) {
#pragma unroll
    for (int half = 0; half < 2; ++half) t[half] = load_angles(a.rope, angle_row, a.rot_dim, u.angle + 4 * half);
  }
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const int h = head0 + i;
    if (h < heads) {
      const __nv_bfloat16* src = copy ? a.v.data + row * a.v.stride_row + h * a.v.stride_head
                                 : h < a.n_q_heads ? a.q.data + row * a.q.stride_row + h * a.q.stride_head
                                                   : a.k.data + row * a.k.stride_row + (h - a.n_q_heads) * a.k.stride_head;
      x[i][0] = load_raw(src + u.first);
      x[i][1] = load_raw(src + u.second);
    }
  }
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const int h = head0 + i;
    if (h < heads) {
      if (BITS == 4 && (copy || h >= a.n_q_heads)) {
        float f[8], g[8];
        widen8(x[i][0], f);
        widen8(x[i][1], g);
        if (turns) {
#pragma unroll
          for (int half = 0; half < 2; ++half) rotate(f, g, t[half], half, a.interleaved);
        }
        const int64_t row4 = cell + (int64_t)(copy ? h : h - a.n_q_heads) * a.kv.block_tokens;
        write_codes<D>((copy ? a.kv.v : a.kv.k) + row4 * (D / 2), (copy ? a.kv.v_scale4 : a.kv.k_scale4) + row4 * (D / kScaleDims), f, g, u, whole);
        continue;
      }
      if (turns) {
        float f[8], g[8];
        widen8(x[i][0], f);
        widen8(x[i][1], g);
#pragma unroll
        for (int half = 0; half < 2; ++half) rotate(f, g, t[half], half, a.interleaved);
        x[i][0] = narrow8(f);
        x[i][1] = narrow8(g);
      }
      __nv_bfloat16* dst;
      if (copy) dst = reinterpret_cast<__nv_bfloat16*>(a.kv.v) + (cell + (int64_t)h * a.kv.block_tokens) * D;
      else if (h < a.n_q_heads) dst = a.q_out.data + row * a.q_out.stride_row + h * a.q_out.stride_head;
      else dst = reinterpret_cast<__nv_bfloat16*>(a.kv.k) + (cell + (int64_t)(h - a.n_q_heads) * a.kv.block_tokens) * D;
      *reinterpret_cast<uint4*>(dst + u.first) = x[i][0];
      *reinterpret_cast<uint4*>(dst + u.second) = x[i][1];
    }
  }
}

// The same for many rows of a 4-bit cache: a warp has a row, all of its heads, four or eight at a time, so that a token's place and angles are
// found once (with a thread for each unit of two heads, 238 instead of 172 us for 54k tokens; with a thread for each unit, as for few rows: 2048 tokens 11.4
// instead of 8.6 us, 1024 7.1 both, 512 4.3 instead of 6.7).  The
// next heads' loads are under way while these are made.
template <int D>
__device__ __forceinline__ void move_whole_rows(const AppendArgs& a, int cta) {
  constexpr int kUnits = D / 16, kHeads = 32 / kUnits, kWarps = kAppendThreads / 32;
  const int row_lo = cta * kWarps, row_hi = min(row_lo + kWarps, a.step.n_rows) - 1, row = row_lo + (int)(threadIdx.x >> 5);
  int lo = 0, hi = 0;
  for (int b = 0; b < a.step.n_seqs; b += kAppendThreads) {
    const int start = b + (int)threadIdx.x < a.step.n_seqs ? __ldg(a.step.row_start + b + threadIdx.x) : 0x7fffffff;
    lo += __syncthreads_count(start <= row_lo);
    hi += __syncthreads_count(start <= row_hi);
  }
  if (row > row_hi || row >= __ldg(a.step.row_start + a.step.n_seqs)) return;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(a.step.row_start + mid) <= row) lo = mid + 1;
    else hi = mid;
  }
  const int seq = lo - 1;
  if (seq < 0) return;
  int pos;
  int64_t angle_row;
  if (!place_of(a, seq, row, &pos, &angle_row)) return;
  const int64_t block = pool_block(a.kv, a.step, seq, pos);
  if (block < 0) {
    report_cache(a.dev_status);
    return;
  }
  const int unit = threadIdx.x % kUnits, first_head = (int)(threadIdx.x & 31) / kUnits;
  const Unit turned = unit_of(unit, a.rope != nullptr ? a.rot_dim : 0, a.interleaved), straight{unit * 16, unit * 16 + 8, -1};
  const int whole = a.rope == nullptr ? 2 : a.rot_dim < D ? 0 : a.interleaved ? 2 : 1;
  Angles t[2];
  if (turned.angle >= 0) {
#pragma unroll
    for (int half = 0; half < 2; ++half) t[half] = load_angles(a.rope, angle_row, a.rot_dim, turned.angle + 4 * half);
  }
  // Heads of one kind: `put` gets the raw or turned elements.
  auto each = [&](const RowsView& rows, int heads, const Unit& u, auto put) {
    const __nv_bfloat16* src = rows.data + row * rows.stride_row + first_head * rows.stride_head;
    const int64_t step = kHeads * rows.stride_head;
    uint4 next[2];
    auto load = [&] {
      next[0] = load_raw(src + u.first);
      next[1] = load_raw(src + u.second);
      src += step;
    };
    if (first_head < heads) load();
#pragma unroll 1
    for (int h = first_head; h < heads; h += kHeads) {
      const uint4 raw[2] = {next[0], next[1]};
      if (h + kHeads < heads) load();
      put(h, raw);
    }
  };
  auto turn_raw = [&](const uint4 (&raw)[2], float (&f)[8], float (&g)[8]) {
    widen8(raw[0], f);
    widen8(raw[1], g);
    if (turned.angle >= 0) {
#pragma unroll
      for (int half = 0; half < 2; ++half) rotate(f, g, t[half], half, a.interleaved);
    }
  };
  const int64_t cell = block * a.kv.n_kv_heads * a.kv.block_tokens + pos % a.kv.block_tokens;
  auto put_codes = [&](uint8_t* pool, uint16_t* scales, int h, const float (&f)[8], const float (&g)[8], const Unit& u, int form) {
    const int64_t at = cell + (int64_t)h * a.kv.block_tokens;
    write_codes<D>(pool + at * (D / 2), scales + at * (D / kScaleDims), f, g, u, form);
  };
  each(a.k, a.kv.n_kv_heads, turned, [&](int h, const uint4 (&raw)[2]) {
    float f[8], g[8];
    turn_raw(raw, f, g);
    put_codes(a.kv.k, a.kv.k_scale4, h, f, g, turned, whole);
  });
  each(a.v, a.kv.n_kv_heads, straight, [&](int h, const uint4 (&raw)[2]) {
    float f[8], g[8];
    widen8(raw[0], f);
    widen8(raw[1], g);
    put_codes(a.kv.v, a.kv.v_scale4, h, f, g, straight, 2);
  });
  each(a.q, a.n_q_heads, turned, [&](int h, const uint4 (&raw)[2]) {
    __nv_bfloat16* dst = a.q_out.data + row * a.q_out.stride_row + h * a.q_out.stride_head;
    uint4 x[2] = {raw[0], raw[1]};
    if (turned.angle >= 0) {
      float f[8], g[8];
      turn_raw(raw, f, g);
      x[0] = narrow8(f), x[1] = narrow8(g);
    }
    *reinterpret_cast<uint4*>(dst + turned.first) = x[0];
    *reinterpret_cast<uint4*>(dst + turned.second) = x[1];
  });
}

// ---------------------------------------------------------------------------------------------- 8-bit groups
// The smallest power of two s >= 2^-100 with m / s <= 448 (448 = 1.75 * 2^8), m finite and not negative.
__device__ __forceinline__ float scale_for(float m) {
  const uint32_t bits = __float_as_uint(m);
  const int exponent = (int)(bits >> 23) - 127;
  const int e = max(exponent - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), -100);
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Four values as E4M3 bytes, to nearest, clipped at 448 (NaN: 0x7F).
__device__ __forceinline__ uint32_t e4m3_four(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n.reg .b16 lo, hi;\ncvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\nmov.b32 %0, {lo, hi};\n}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ float2 e4m3_pair_value(uint32_t two) {
  uint32_t h2;
  asm("{\n.reg .b16 b;\ncvt.u16.u32 b, %1;\ncvt.rn.f16x2.e4m3x2 %0, b;\n}" : "=r"(h2) : "r"(two));
  return __half22float2(*reinterpret_cast<const __half2*>(&h2));
}

__device__ __forceinline__ uint2 bytes8(const float (&x)[8], float inverse) {
  return make_uint2(e4m3_four(x[0] * inverse, x[1] * inverse, x[2] * inverse, x[3] * inverse),
                    e4m3_four(x[4] * inverse, x[5] * inverse, x[6] * inverse, x[7] * inverse));
}

__device__ __forceinline__ float finite_magnitude(float x) {
  const float m = fabsf(x);
  return m <= 3.402823466e38f ? m : 0.f;            // neither infinities nor NaN set a scale
}
// Largest of `top` and the magnitudes, those that are not finite apart if FINITE (else NaN only).
template <bool FINITE>
__device__ __forceinline__ float largest(const float (&x)[2][8], float top) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 8; e += 2)
      top = FINITE ? fmaxf(top, fmaxf(finite_magnitude(x[h][e]), finite_magnitude(x[h][e + 1]))) : max3(top, fabsf(x[h][e]), fabsf(x[h][e + 1]));
  return top;
}
// The largest of all threads' values.
__device__ __forceinline__ float largest_of_cta(float top, float* warp_max) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  __syncthreads();                                  // of values of another call, and of what was read before it
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kAppendThreads / 32; ++w) top = fmaxf(top, warp_max[w]);
  return top;
}

// A group of 64 tokens (of a sequence, in a pool block): keys and values of some of its heads in turn; while ones are made, the next
// ones' rows are on their way.  Group slots of the grid: sequence b owns those from row_start[b] / 64 + 2 b on, which is at
// least as many as its new tokens can touch (n tokens touch at most n / 64 + 2 groups).
template <int D, bool MANY>
__device__ __forceinline__ void fill_group(const AppendArgs& a, int index) {
  constexpr int kUnits = D / 16, kPer = kScaleTokens * kUnits / kAppendThreads;
  __shared__ float warp_max[kAppendThreads / 32];
  // a CTA's share of the group: keys and values of some heads, or one head's keys or values
  const int pieces = MANY ? (a.kv.n_kv_heads + a.fill_heads - 1) / a.fill_heads : 2 * a.kv.n_kv_heads;
  const int slot = index / pieces, piece = index - slot * pieces;
  const bool only_v = !MANY && piece >= a.kv.n_kv_heads;
  const int head0 = MANY ? piece * a.fill_heads : only_v ? piece - a.kv.n_kv_heads : piece, head1 = min(head0 + (MANY ? a.fill_heads : 1), a.kv.n_kv_heads);
  int count = 0;
  for (int b = 0; b < a.step.n_seqs; b += kAppendThreads) {
    const int at = b + (int)threadIdx.x;
    count += __syncthreads_count(at < a.step.n_seqs && __ldg(a.step.row_start + min(at, a.step.n_seqs)) / kScaleTokens + 2 * at <= slot);
  }
  const int seq = count - 1;
  if (seq < 0) return;
  const int start = __ldg(a.step.row_start + seq), behind = __ldg(a.step.row_start + seq + 1), len = __ldg(a.step.seq_lens + seq);
  const int end = min(behind, a.step.n_rows);
  const int old_len = place_from_end(len, (int64_t)behind - start);      // tokens before the step
  // the group's first token, and its tokens of the step, by position (64 bits: a length may be anything)
  const int64_t from = ((int64_t)(max(old_len, 0) / kScaleTokens) + slot - (start / kScaleTokens + 2 * seq)) * kScaleTokens;
  const int64_t begin = max(from, (int64_t)max(old_len, 0)), upto = min(from + kScaleTokens, min((int64_t)len, (int64_t)old_len + end - start));
  const int first = (int)from, lo = (int)begin, hi = (int)upto;
  if (start < 0 || begin >= upto) {
    if (threadIdx.x == 0 && old_len < 0) report_cache(a.dev_status);
    return;
  }
  const int64_t block = pool_block(a.kv, a.step, seq, first);
  if (block < 0 || old_len < 0) {
    if (threadIdx.x == 0) report_cache(a.dev_status);
    if (block < 0) return;
  }
  const int off = first % a.kv.block_tokens;

  // the thread's units: unit threadIdx.x mod units of every (threads / units)-th token
  const int unit = threadIdx.x % kUnits, token0 = threadIdx.x / kUnits;
  constexpr int kTokenStep = kAppendThreads / kUnits;
  const int row0 = start + (first + token0 - old_len);
  bool live[kPer];
  int angle_row[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int pos = first + token0 + i * kTokenStep;
    live[i] = pos >= lo && pos < hi;
    angle_row[i] = pos;
    if (live[i] && a.rope != nullptr) {
      if (a.positions != nullptr) angle_row[i] = __ldg(a.positions + row0 + i * kTokenStep);
      if (angle_row[i] < 0 || angle_row[i] >= a.n_positions) {
        live[i] = false;
        report_cache(a.dev_status);
      }
    }
  }
  const Unit turned = unit_of(unit, a.rope != nullptr ? a.rot_dim : 0, a.interleaved), straight{unit * 16, unit * 16 + 8, -1};
  auto fetch = [&](const __nv_bfloat16* src, int64_t stride_row, const Unit& u, uint4 (&raw)[kPer][2]) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      raw[i][0] = raw[i][1] = make_uint4(0, 0, 0, 0);
      if (live[i]) {
        raw[i][0] = load_raw(src + i * kTokenStep * stride_row + u.first);
        raw[i][1] = load_raw(src + i * kTokenStep * stride_row + u.second);
      }
    }
  };
  const __nv_bfloat16* k_src = a.k.data + row0 * a.k.stride_row + head0 * a.k.stride_head;
  const __nv_bfloat16* v_src = a.v.data + row0 * a.v.stride_row + head0 * a.v.stride_head;
  // places of the thread's first token and of the group's scale in the pools, the same for keys and values
  int64_t cell = ((block * a.kv.n_kv_heads + head0) * a.kv.block_tokens + off) * D;
  int64_t scale_cell = (block * a.kv.n_kv_heads + head0) * (a.kv.block_tokens / kScaleTokens) + off / kScaleTokens;
  const bool partly = lo > first;                   // the group holds tokens from before the step
  uint4 raw[kPer][2];
  // The thread's angles wait in shared memory, where their copy is on its way with the first rows: in registers there is no room, and
  // loaded when the rows are there they are waited for once more.
  __shared__ float4 angles[kPer][4][kAppendThreads];
  const bool with_angles = !only_v && turned.angle >= 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (with_angles && live[i]) {
      const float* at = a.rope + (int64_t)angle_row[i] * a.rot_dim + turned.angle;
#pragma unroll
      for (int j = 0; j < 4; ++j) copy_async(smem_u32(&angles[i][j][threadIdx.x]), at + (j >> 1) * (a.rot_dim / 2) + 4 * (j & 1));
    }
  }

  // Makes the bytes of what `raw` holds; `next` fetches the rows after these.
  auto fill = [&](auto is_v, auto next) {
    constexpr bool kValues = decltype(is_v)::value;
    uint8_t* cells = (kValues ? a.kv.v : a.kv.k) + cell;
    float* scale_at = (kValues ? a.kv.v_scale : a.kv.k_scale) + scale_cell;
    const Unit u = kValues ? straight : turned;
    const float held = partly ? *scale_at : 0.f;    // every thread has it before one of them writes the new one: barriers follow
    float x[kPer][2][8];
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      widen8(raw[i][0], x[i][0]);
      widen8(raw[i][1], x[i][1]);
    }
    next();
    if (!kValues) asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (!kValues && with_angles && live[i]) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
          rotate(x[i][0], x[i][1], Angles{angles[i][half][threadIdx.x], angles[i][2 + half][threadIdx.x]}, half, a.interleaved);
      }
      top = largest<false>(x[i], top);              // rows that are not there are zeros
    }
    top = largest_of_cta(top, warp_max);
    if (!(top <= 3.402823466e38f)) {
      top = 0.f;                                    // some are infinite: once more without them
#pragma unroll
      for (int i = 0; i < kPer; ++i) top = largest<true>(x[i], top);
      top = largest_of_cta(top, warp_max);
    }
    const float scale = fmaxf(held, scale_for(top));
    if (threadIdx.x == 0 && scale != held) *scale_at = scale;
    // x / scale is a product where the scale is a power of two (whose inverse is one too), as every scale that this kernel makes; else
    // the quotients are made here
    const uint32_t bits = __float_as_uint(scale);
    float inverse = __uint_as_float((254u << 23) - bits);
    if ((bits & 0x7fffffu) != 0 || bits >= 254u << 23) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[i][0][e] = __fdiv_rn(x[i][0][e], scale);
          x[i][1][e] = __fdiv_rn(x[i][1][e], scale);
        }
      inverse = 1.f;
    }
    if (partly && scale != held) {
      const float ratio = __fdiv_rn(held, scale);
      for (int i = threadIdx.x; i < (lo - first) * (D / 16); i += kAppendThreads) {
        uint4* at = reinterpret_cast<uint4*>(cells) + i;
        uint4 v = *at;
        uint32_t* w = &v.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 p = e4m3_pair_value(w[j] & 0xffffu), r = e4m3_pair_value(w[j] >> 16);
          w[j] = e4m3_four(p.x * ratio, p.y * ratio, r.x * ratio, r.y * ratio);
        }
        *at = v;
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (!live[i]) continue;
      uint8_t* dst = cells + (token0 + i * kTokenStep) * D;
      *reinterpret_cast<uint2*>(dst + u.first) = bytes8(x[i][0], inverse);
      *reinterpret_cast<uint2*>(dst + u.second) = bytes8(x[i][1], inverse);
    }
  };
  const std::integral_constant<bool, false> keys;
  const std::integral_constant<bool, true> values;
  if constexpr (!MANY) {
    if (only_v) {
      fetch(v_src, a.v.stride_row, straight, raw);
      fill(values, [] {});
    } else {
      fetch(k_src, a.k.stride_row, turned, raw);
      fill(keys, [] {});
    }
  } else {
    fetch(k_src, a.k.stride_row, turned, raw);
    for (int head = head0; head < head1; ++head) {
      fill(keys, [&] { fetch(v_src, a.v.stride_row, straight, raw); });
      k_src += a.k.stride_head;
      v_src += a.v.stride_head;
      fill(values, [&] {
        if (head + 1 < head1) fetch(k_src, a.k.stride_row, turned, raw);
      });
      cell += (int64_t)a.kv.block_tokens * D;
      scale_cell += a.kv.block_tokens / kScaleTokens;
    }
  }
}

template <int D, int HPT, int BITS>
__global__ void __launch_bounds__(kAppendThreads, BITS == 8 ? 3 : 4) append_kernel(const __grid_constant__ AppendArgs a) {
  const int fills = (int)gridDim.x - a.rotate_ctas;
  if (BITS == 4 && HPT > 1) move_whole_rows<D>(a, (int)blockIdx.x);
  else if (BITS == 8 && (int)blockIdx.x < fills) fill_group<D, (HPT > 1)>(a, (int)blockIdx.x);
  else move_rows<D, HPT, BITS>(a, (int)blockIdx.x - (BITS == 8 ? fills : 0));
}

template <int D, int BITS>
int32_t launch_append(AppendArgs& a, cudaStream_t stream) {
  constexpr bool FP8 = BITS == 8;
  const int turned = a.n_q_heads + (FP8 ? 0 : a.kv.n_kv_heads), copied = FP8 ? 0 : a.kv.n_kv_heads;
  // Few rows: a head to a thread, a head's keys or values of a group to a CTA, so that everything is under way at once.  Where that
  // more than fills the chip: two heads to a thread, which read a row's angles once, and keys and values of several heads of a group to
  // a CTA, which finds its place once, keeps the angles and fetches the next rows while it makes these.
  const int64_t slots = FP8 ? a.step.n_rows / kScaleTokens + 2 * (int64_t)a.step.n_seqs : 0, lanes = 2 * (int64_t)a.kv.n_kv_heads;
  const bool many = (int64_t)a.step.n_rows * (a.n_q_heads + lanes) * (D / 16) > 148 * 2048;
  const int hpt = many ? 2 : 1;
  const int64_t items = (int64_t)a.step.n_rows * (ceil_div(turned, hpt) + ceil_div(copied, hpt)) * (D / 16);
  // Eight such heads, fewer where that would leave SMs without a CTA.  8 heads of 128 dimensions: 54k tokens 198 us (with two heads 210),
  // 8192 tokens 27.8 (wanting three CTAs an SM 29.5, half of one 33.2), 4096 tokens 13.0 (14.7, 14.2).
  a.fill_heads = 8;
  while (a.fill_heads > 1 && slots * ceil_div(a.kv.n_kv_heads, a.fill_heads) < 148) a.fill_heads /= 2;
  int64_t rotate = ceil_div(items, kAppendThreads);
  const int64_t groups = slots * (many ? ceil_div(a.kv.n_kv_heads, a.fill_heads) : lanes);
  if (rotate + groups > 0x7fffffffLL) return fail(SPF_ERR_UNSUPPORTED, "spf_kv_append: too many rows for one launch");
  if (rotate + groups == 0) return SPF_OK;
  if (BITS == 4 && many) rotate = ceil_div(a.step.n_rows, kAppendThreads / 32);
  a.rotate_ctas = (int)rotate;
  const int64_t per_row = (ceil_div(turned, hpt) + ceil_div(copied, hpt)) * (D / 16);
  if (per_row >= (1 << 20)) return fail(SPF_ERR_UNSUPPORTED, "spf_kv_append: too many heads");
  a.per_row_inverse = per_row > 0 ? ~0ull / (uint64_t)per_row + 1 : 0;
  if (many) append_kernel<D, 2, BITS><<<(unsigned)(rotate + groups), kAppendThreads, 0, stream>>>(a);
  else append_kernel<D, 1, BITS><<<(unsigned)(rotate + groups), kAppendThreads, 0, stream>>>(a);
  SPF_CUDA_CHECK(cudaGetLastError());
  return SPF_OK;
}

}  // namespace

int32_t check_cache(const char* who, const spf_kv_cache* c, KvView* out) {
  if (c == nullptr) return fail(SPF_ERR_INVALID_ARG, "%s: cache is null", who);
  if (c->k_pool == nullptr || c->v_pool == nullptr) return fail(SPF_ERR_INVALID_ARG, "%s: k_pool or v_pool is null", who);
  if ((c->k_scale == nullptr) != (c->v_scale == nullptr))
    return fail(SPF_ERR_INVALID_ARG, "%s: k_scale and v_scale are both given (8-bit and 4-bit pools) or both null (bf16 pools)", who);
  if (c->bits != 0 && c->bits != 4 && c->bits != 8 && c->bits != 16) return fail(SPF_ERR_INVALID_ARG, "%s: bits must be 4, 8, 16 or 0 (got %d)", who, c->bits);
  const int bits = cache_bits(c);
  if ((bits == 16) != (c->k_scale == nullptr)) return fail(SPF_ERR_INVALID_ARG, "%s: pools of 4 and 8 bits have scales, bf16 pools none", who);
  if (reinterpret_cast<uintptr_t>(c->k_pool) % 16 != 0 || reinterpret_cast<uintptr_t>(c->v_pool) % 16 != 0)
    return fail(SPF_ERR_INVALID_ARG, "%s: k_pool or v_pool is not 16-byte aligned", who);
  const uintptr_t aligned = bits == 4 ? 16 : 4;
  if (reinterpret_cast<uintptr_t>(c->k_scale) % aligned != 0 || reinterpret_cast<uintptr_t>(c->v_scale) % aligned != 0)
    return fail(SPF_ERR_INVALID_ARG, "%s: k_scale or v_scale is not %d-byte aligned", who, (int)aligned);
  if (c->n_pool_blocks < 1 || c->n_kv_heads < 1) return fail(SPF_ERR_INVALID_ARG, "%s: the pool has no blocks or no heads", who);
  if (c->block_tokens < 128 || c->block_tokens % 128 != 0)
    return fail(SPF_ERR_INVALID_ARG, "%s: block_tokens must be a positive multiple of 128 (got %d)", who, c->block_tokens);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(SPF_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128 (got %d)", who, c->head_dim);
  const int64_t per_block = (int64_t)c->n_kv_heads * c->block_tokens;
  if (per_block > 0x7fffffffLL || c->n_pool_blocks > 0x7fffffffLL / per_block)
    return fail(SPF_ERR_UNSUPPORTED, "%s: n_pool_blocks * n_kv_heads * block_tokens is 2^31 or more", who);
  *out = KvView{static_cast<uint8_t*>(c->k_pool), static_cast<uint8_t*>(c->v_pool), nullptr, nullptr, nullptr, nullptr, c->n_pool_blocks,
                c->block_tokens, c->n_kv_heads, bits};
  if (bits == 8) out->k_scale = static_cast<float*>(c->k_scale), out->v_scale = static_cast<float*>(c->v_scale);
  if (bits == 4) out->k_scale4 = static_cast<uint16_t*>(c->k_scale), out->v_scale4 = static_cast<uint16_t*>(c->v_scale);
  return SPF_OK;
}

int32_t check_step(const char* who, const spf_kv_step* s, StepView* out) {
  if (s == nullptr) return fail(SPF_ERR_INVALID_ARG, "%s: step is null", who);
  if (s->n_seqs < 1 || s->n_seqs > (1 << 20) || s->n_rows < 0 || s->n_rows > (1 << 30) || s->max_new < 1 || s->table_stride < 1)
    return fail(SPF_ERR_INVALID_ARG, "%s: n_seqs, max_new and table_stride must be positive (n_seqs at most 2^20), n_rows in [0, 2^30]", who);
  if (s->row_start == nullptr || s->seq_lens == nullptr || s->block_table == nullptr)
    return fail(SPF_ERR_INVALID_ARG, "%s: row_start, seq_lens or block_table is null", who);
  *out = StepView{s->row_start, s->seq_lens, s->block_table, s->n_seqs, s->n_rows, s->table_stride};
  return SPF_OK;
}

int32_t check_rows(const char* who, const char* name, const spf_rows* r, int n_heads, int head_dim, bool written, RowsView* out) {
  if (r == nullptr || r->data == nullptr) return fail(SPF_ERR_INVALID_ARG, "%s: %s is null", who, name);
  if (reinterpret_cast<uintptr_t>(r->data) % 16 != 0) return fail(SPF_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", who, name);
  if (r->stride_row % 8 != 0 || r->stride_head % 8 != 0 || r->stride_row < 0 || r->stride_head < 0)
    return fail(SPF_ERR_INVALID_ARG, "%s: the strides of %s must be multiples of 8, not negative", who, name);
  if (written && (r->stride_row < head_dim || (n_heads > 1 && r->stride_head < head_dim)))
    return fail(SPF_ERR_INVALID_ARG, "%s: heads or rows of %s overlap", who, name);
  *out = RowsView{static_cast<__nv_bfloat16*>(r->data), r->stride_row, r->stride_head};
  return SPF_OK;
}

// Slices of one buffer lie in one range of memory without meeting, so ranges alone decide only where they are apart.  Else each run of a's
// elements is held against b's rows: of a row i of b, of w elements, [i S, i S + w), the first that ends behind the run's start decides.
// With equal strides of rows (slices of one buffer) one row of a stands for all, rows of b before it being negative ones.
bool rows_meet(const RowsView& a, int a_heads, const RowsView& b, int b_heads, int n_rows, int head_dim) {
  struct Runs {
    int64_t heads, width, stride_head, extent;
  };
  const int64_t rows = n_rows;
  auto runs_of = [&](const RowsView& v, int heads) {
    const bool joined = heads == 1 || v.stride_head == head_dim;       // a row's heads are one run
    return Runs{joined ? 1 : heads, joined ? (int64_t)heads * head_dim : head_dim, v.stride_head, (rows - 1) * v.stride_row + (heads - 1) * v.stride_head + head_dim};
  };
  const Runs ra = runs_of(a, a_heads), rb = runs_of(b, b_heads);
  const int64_t apart = (int64_t)(reinterpret_cast<intptr_t>(a.data) - reinterpret_cast<intptr_t>(b.data)) / (int64_t)sizeof(__nv_bfloat16);
  if (apart >= rb.extent || apart + ra.extent <= 0) return false;
  const bool same = a.stride_row == b.stride_row;
  for (int64_t r = 0; r < (same || a.stride_row == 0 ? 1 : rows); ++r)
    for (int64_t h = 0; h < ra.heads; ++h)
      for (int64_t g = 0; g < rb.heads; ++g) {
        const int64_t x = apart + r * a.stride_row + h * ra.stride_head - g * rb.stride_head, y = x - rb.width, S = b.stride_row;   // S > 0: b is written
        const int64_t first = std::max((y >= 0 ? y / S : -((-y + S - 1) / S)) + 1, same ? 1 - rows : 0);
        if (first < rows && first * S < x + ra.width) return true;
      }
  return false;
}

}  // namespace spf

using namespace spf;

extern "C" int32_t spf_kv_append(const spf_kv_cache* cache, const spf_kv_step* step, const spf_rope* rope, const spf_rows* k,
                                 const spf_rows* v, const spf_rows* q, const spf_rows* q_out, int32_t n_q_heads,
                                 int32_t* dev_status, void* cuda_stream) {
  const char* who = "spf_kv_append";
  clear_error();
  AppendArgs a{};
  int32_t st = check_cache(who, cache, &a.kv);
  if (st == SPF_OK) st = check_step(who, step, &a.step);
  if (st == SPF_OK && step->n_rows == 0) return SPF_OK;
  if (st == SPF_OK) st = check_rows(who, "k", k, cache->n_kv_heads, cache->head_dim, false, &a.k);
  if (st == SPF_OK) st = check_rows(who, "v", v, cache->n_kv_heads, cache->head_dim, false, &a.v);
  if (st != SPF_OK) return st;
  if ((q == nullptr) != (q_out == nullptr)) return fail(SPF_ERR_INVALID_ARG, "%s: q and q_out are both given or both null", who);
  if (q != nullptr) {
    if (n_q_heads < 1) return fail(SPF_ERR_INVALID_ARG, "%s: n_q_heads must be positive", who);
    st = check_rows(who, "q", q, n_q_heads, cache->head_dim, false, &a.q);
    if (st == SPF_OK) st = check_rows(who, "q_out", q_out, n_q_heads, cache->head_dim, true, &a.q_out);
    if (st != SPF_OK) return st;
    const bool in_place = q->data == q_out->data && q->stride_row == q_out->stride_row && q->stride_head == q_out->stride_head;
    if (!in_place && rows_meet(a.q, n_q_heads, a.q_out, n_q_heads, step->n_rows, cache->head_dim))
      return fail(SPF_ERR_INVALID_ARG, "%s: q_out overlaps q and is not q", who);
    if (rows_meet(a.k, cache->n_kv_heads, a.q_out, n_q_heads, step->n_rows, cache->head_dim) ||
        rows_meet(a.v, cache->n_kv_heads, a.q_out, n_q_heads, step->n_rows, cache->head_dim))
      return fail(SPF_ERR_INVALID_ARG, "%s: q_out overlaps k or v", who);
    a.n_q_heads = n_q_heads;
  }
  if (rope != nullptr) {
    if (rope->table == nullptr || reinterpret_cast<uintptr_t>(rope->table) % 16 != 0)
      return fail(SPF_ERR_INVALID_ARG, "%s: the rotation's table is null or not 16-byte aligned", who);
    if (rope->n_positions < 1 || rope->rot_dim < 16 || rope->rot_dim % 16 != 0 || rope->rot_dim > cache->head_dim)
      return fail(SPF_ERR_INVALID_ARG, "%s: rot_dim must be a multiple of 16 in [16, head_dim] and n_positions positive", who);
    a.rope = rope->table;
    a.positions = rope->positions;
    a.n_positions = rope->n_positions;
    a.rot_dim = rope->rot_dim;
    a.interleaved = rope->interleaved != 0;
  }
  a.dev_status = dev_status;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool d64 = cache->head_dim == 64;
  switch (a.kv.bits) {
    case 4: return d64 ? launch_append<64, 4>(a, stream) : launch_append<128, 4>(a, stream);
    case 8: return d64 ? launch_append<64, 8>(a, stream) : launch_append<128, 8>(a, stream);
    default: return d64 ? launch_append<64, 16>(a, stream) : launch_append<128, 16>(a, stream);
  }
}
