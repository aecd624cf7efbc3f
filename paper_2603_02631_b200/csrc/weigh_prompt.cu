// The attention weights that the cache's tokens receive from a step with many rows per key head (chunks of prompts).
//
//   W[h, s] = decay W[h, s] + sum over rows r that see s of 2^(f_s q[r] . k[s] - lse2[r])
//
// A weight is one product of D dimensions and one exponential, and the exponentials bound it: 128 keys by 128 rows take the exponential unit
// 1024 cycles, the tensor cores 128 (64 dimensions) or 256.  So the products are the big instruction's, into tensor memory, with keys as the 128
// lanes and rows as the columns: a thread of the four sets of four warps that take the exponentials has one key, whose weights it adds up in a
// register over all rows, with no exchange between threads; per exponential it spends half a multiply-add, half an addition and a quarter of a
// read of log-sum-exps from shared memory.  Three chunks of 836 to 2001 tokens behind 1300 to 9000 (32/8 heads of 64 dimensions, 8 bits) take
// 340 us, 222 of them exponentials; warp-level products with keys in registers took 648: two units in turns in each of few warps.  Two sets of
// warps for the exponentials instead of four: 385; rows brought by threads instead of tensor copies: 405, log-sum-exps loaded one tile at a time:
// 447.  Sums of tiles are added with what the additions lose (thousands of rows make 1.7e-6 of a weight otherwise).
//
// Keys are brought once for all rows of an item (a sequence, key head and 128 keys), eight loads in flight, and widened to bf16 on the way (exactly: 8-bit values, and
// 4-bit codes times scales of five bits), the next item's while this one's last rows are being made.  Rows go by in tiles of as many tokens as fit whole into 128, a box of the queries each, whose
// strides the tensor map has.
//
// The list of all items, each as long as the tiles of rows that see any of its keys, is cut into one part for each SM; an item belongs to the
// part that its beginning lies in.
//
// Warps: sets of four for the exponentials, a tile each in turn; four for keys and log-sum-exps; one issues the products, one copies rows.
#include <climits>

#include "weigh.cuh"

namespace spf {
namespace {

constexpr int kSets = 4, kThreads = (4 * kSets + 6) * 32, kKeys = 128, kEnds = 4;
constexpr int kAccs = 4, kBelow = 16;                     // accumulators in tensor memory; tiles whose log-sum-exps are kept: more than may be under way

template <int D_, int BITS_>
struct Traits {
  static constexpr int D = D_, BITS = BITS_, TILE = 128 * D * 2, STAGES = D == 64 ? 6 : 4;
};

struct Smem {
  unsigned long long q_full[6], q_empty[6], b_full[6], k_full[2], k_empty[2], acc_full[kAccs], acc_empty[kAccs], summed, mma_done;
  float below[kBelow][128];                             // the rows' base-2 log-sum-exps, negated
  float sums[2][kSets - 1][kKeys];                        // of all sets but the first
  int64_t scan[kThreads / 32];
  int64_t total, start_base;
  int start_seq;
  int abort;
  int idle;                                             // some row of the CTA's saw no key
  uint32_t tmem;
};

template <class T>
constexpr int smem_bytes() { return (2 + T::STAGES) * T::TILE + (int)sizeof(Smem) + 1024; }

// ---------------------------------------------------------------------------------------------- the list of items
// Tokens whose rows make a tile: as many as fit whole.
__device__ __forceinline__ int tile_tokens(const WeighArgs& w) { return 128 / w.a.group; }
// Of a sequence's tokens the first that sees key0.
__device__ __forceinline__ int first_token(const WeighArgs& w, const SeqSpan& s, int key0) {
  return w.a.causal ? (int)min(max((int64_t)key0 - s.pos0, (int64_t)0), (int64_t)s.n_new) : 0;
}
__device__ __forceinline__ int tiles_of(const WeighArgs& w, const SeqSpan& s, int key0) {
  if (key0 + kKeys <= s.first) return 0;
  return (s.n_new - first_token(w, s, key0) + tile_tokens(w) - 1) / tile_tokens(w);
}
// Length of a (sequence, key head) in the list: its tiles of rows, and for an item's beginning and end as long as kEnds of them.
__device__ __forceinline__ int64_t head_cost(const WeighArgs& w, const SeqSpan& s) {
  const int tiles = (s.end + kKeys - 1) / kKeys;
  // keys before the first that every row sees, and those from the first row's on
  const int before = s.first / kKeys, all = w.a.causal ? min(max(s.pos0, 0) / kKeys, tiles) : tiles;
  int64_t cost = (int64_t)kEnds * tiles;
  if (all > before) cost += (int64_t)(all - before) * tiles_of(w, s, before * kKeys);
  for (int t = max(all, before); t < tiles; ++t) cost += tiles_of(w, s, t * kKeys);
  return cost;
}

struct Cursor {
  int seq, head, tile;
  int64_t at;                     // where the item begins in the list
};

// Length of the list, and the sequence that holds the CTA's beginning.
__device__ __forceinline__ void find_start(const WeighArgs& w, Smem& sm) {
  const int n_seqs = w.a.step.n_seqs, run = (n_seqs + kThreads - 1) / kThreads, lo = min((int)threadIdx.x * run, n_seqs), hi = min(lo + run, n_seqs);
  auto cost_of = [&](int b) {
    const WeighSpan s = weigh_span(w, b);
    return s.rows.n_new > 0 ? w.a.kv.n_kv_heads * head_cost(w, s.rows) : 0;
  };
  int64_t mine = 0;
  for (int b = lo; b < hi; ++b) mine += cost_of(b);
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
  for (int i = 0; i < kThreads / 32; ++i) {
    if (i < warp) upto += sm.scan[i];
    total += sm.scan[i];
  }
  const int64_t w0 = (total + gridDim.x - 1) / gridDim.x * blockIdx.x;
  if (threadIdx.x == 0) sm.total = total;
  if (w0 >= upto - mine && w0 < upto) {
    int64_t base = upto - mine;
    int b = lo;
    for (; b < hi - 1; ++b) {
      const int64_t c = cost_of(b);
      if (w0 < base + c) break;
      base += c;
    }
    sm.start_seq = b;
    sm.start_base = base;
  }
  __syncthreads();
}

// The first item that begins at w0 or behind it.
__device__ __forceinline__ Cursor first_item(const WeighArgs& w, const Smem& sm, int64_t w0) {
  Cursor c{sm.start_seq, 0, 0, sm.start_base};
  const SeqSpan s = weigh_span(w, c.seq).rows;
  const int64_t per_head = head_cost(w, s);
  c.head = (int)((w0 - c.at) / per_head);
  c.at += c.head * per_head;
  const int tiles = (s.end + kKeys - 1) / kKeys, before = s.first / kKeys, all = w.a.causal ? min(max(s.pos0, 0) / kKeys, tiles) : tiles;
  if (all > before && w0 > c.at + kEnds * before) {
    // among the items of equal length, without looking at each
    const int64_t each = tiles_of(w, s, before * kKeys) + kEnds, skip = min((w0 - c.at - kEnds * before) / each, (int64_t)(all - before));
    c.tile = before + (int)skip;
    c.at += kEnds * before + skip * each;
  }
  while (c.at < w0) c.at += tiles_of(w, s, c.tile++ * kKeys) + kEnds;
  return c;
}

// A CTA's items one after the other, as every role walks through them.
struct Walk {
  Cursor at;
  WeighSpan span;
  int64_t end;
  int key0, tiles, token;                                 // of the item; token: the first of its first tile
  int pool_at;                                            // the first key's row in the pool
  bool inside;

  __device__ __forceinline__ Walk(const WeighArgs& w, const Smem& sm, int64_t w0, int64_t w1) : at(first_item(w, sm, w0)), span(weigh_span(w, at.seq)), end(w1) {}
  __device__ __forceinline__ bool next(const WeighArgs& w) {
    if (at.at >= end) return false;
    while (span.rows.n_new <= 0 || at.tile * kKeys >= span.rows.end) {
      at.tile = 0;
      if (span.rows.n_new <= 0 || span.rows.end == 0 || ++at.head >= w.a.kv.n_kv_heads) {
        at.head = 0;
        if (++at.seq >= w.a.step.n_seqs) return false;
        span = weigh_span(w, at.seq);
      }
    }
    key0 = at.tile * kKeys;
    tiles = tiles_of(w, span.rows, key0);
    token = first_token(w, span.rows, key0);
    pool_at = pool_row(w.a, at.seq, at.head, key0);
    inside = pool_at < w.a.kv.n_blocks * w.a.kv.n_kv_heads * w.a.kv.block_tokens;
    at.at += tiles + kEnds;
    ++at.tile;
    return true;
  }
};

// ---------------------------------------------------------------------------------------------- keys
__device__ __forceinline__ uint32_t mul_bf16(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Eight elements of a key from dimension 8 j on as the cache has them (`row`: the key's row in the pool), and as bf16 pairs.
template <class T>
struct Eight {
  uint32_t raw[T::BITS / 4];
  uint32_t scale;                                         // 4 bits

  __device__ __forceinline__ void load(const KvView& kv, int64_t row, int j) {
    if constexpr (T::BITS == 16) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(kv.k + row * (2 * T::D)) + j);
      raw[0] = v.x, raw[1] = v.y, raw[2] = v.z, raw[3] = v.w;
    } else if constexpr (T::BITS == 8) {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(kv.k + row * T::D) + j);
      raw[0] = v.x, raw[1] = v.y;
    } else {
      raw[0] = __ldg(reinterpret_cast<const uint32_t*>(kv.k + row * (T::D / 2)) + j);
      scale = __ldg(kv.k_scale4 + row * (T::D / kScaleDims) + j / 4);
    }
  }
  __device__ __forceinline__ uint4 widen() const {
    uint32_t r[4];
    if constexpr (T::BITS == 16) {
      return make_uint4(raw[0], raw[1], raw[2], raw[3]);
    } else if constexpr (T::BITS == 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t two = __byte_perm(raw[i / 2], 0, i & 1 ? 0x4342 : 0x4140);
        // a byte s eeee mmm at the bits s 0000eeee mmm0000 is its value times 2^-120
        r[i] = mul_bf16(((two << 8) & 0x80008000u) | ((two << 4) & 0x07f007f0u), 0x7b807b80u);
      }
      if (((((raw[0] & 0x7f7f7f7fu) + 0x01010101u) | ((raw[1] & 0x7f7f7f7fu) + 0x01010101u)) & 0x80808080u) != 0) {
        // NaN, which looks like 480
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (((raw[i / 4] >> (8 * (i & 3))) & 0x7fu) == 0x7fu) r[i / 2] |= 0x7fffu << (16 * (i & 1));
      }
    } else {
      const uint32_t both = scale | scale << 16, less = mul_bf16(both, 0xc1c0c1c0u);                                          // -24 scales
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t two = raw[0] >> (8 * i);
        r[i] = ((two & 0xfu) << 3) | ((two & 0xf0u) << 15) | 0x41804180u;                                                      // 16 + code
        asm("fma.rn.bf16x2 %0, %0, %1, %2;" : "+r"(r[i]) : "r"(both), "r"(less));
      }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
  }
};

// ---------------------------------------------------------------------------------------------- keys and rows into shared memory
// The copying thread: a tile of rows is a box of the queries, spans of 64 dimensions x heads of the group x tokens.
template <class T>
__device__ __forceinline__ void copy_rows(const WeighArgs& w, Smem& sm, uint32_t q_ring, int64_t w0, int64_t w1, const Abort& ab) {
  const int tokens = tile_tokens(w);
  const uint32_t bytes = (uint32_t)(tokens * w.a.group * T::D * 2);
  const bool on = elect_one();
  Walk walk(w, sm, w0, w1);
  uint32_t done = 0;
  while (walk.next(w)) {
    for (int j = 0; j < walk.tiles; ++j, ++done) {
      const uint32_t slot = done % T::STAGES, bar = smem_u32(&sm.q_full[slot]);
      if (!mbar_wait_warp(smem_u32(&sm.q_empty[slot]), ((done / T::STAGES) & 1u) ^ 1u, ab)) {
        // a stage's last copy was its (done - stage) / STAGES-th, rounded up
        const uint32_t stage = threadIdx.x & 31;
        if (stage < T::STAGES && done > stage) drain_copy(smem_u32(&sm.q_full[stage]), ((done - stage + T::STAGES - 1) / T::STAGES - 1) & 1u);
        return;
      }
      if (on) {
        mbar_expect_tx(bar, bytes);
#pragma unroll
        for (int x = 0; x < T::D; x += 64)
          tma_load_3d(q_ring + slot * T::TILE + x * 256, &w.q_map, x, walk.at.head * w.a.group, walk.span.rows.row0 + walk.token + j * tokens, bar);
      }
      __syncwarp();
    }
  }
}

// Byte offset of the 16-byte chunk of a row of keys, as the products read them: spans of 128 bytes, swizzled.
__device__ __forceinline__ uint32_t tile_chunk(int row, int chunk) { return (uint32_t)((chunk >> 3) * (128 * 128) + row * 128 + ((chunk ^ row) & 7) * 16); }

// Keys, widened, and log-sum-exps, made what the exponentials want; those of four tiles are loaded together.
template <class T>
__device__ __forceinline__ void bring(const WeighArgs& w, Smem& sm, unsigned char* k_tiles, int64_t w0, int64_t w1, const Abort& ab) {
  constexpr int kChunks = T::D / 8, kLines = 128 / kChunks, kAhead = 4;
  const AttendArgs& a = w.a;
  const int thread = (int)threadIdx.x - 128 * kSets, lane = threadIdx.x & 31, first = thread / kChunks, chunk = thread % kChunks;
  const int tokens = tile_tokens(w), own_token = thread / a.group, own_head = thread - own_token * a.group;
  Walk walk(w, sm, w0, w1);
  uint32_t done = 0, items = 0;                           // tiles and items brought
  while (walk.next(w)) {
    if (walk.tiles == 0) continue;
    const SeqSpan& s = walk.span.rows;
    const uint32_t buf = items & 1u;
    if (!mbar_wait_warp(smem_u32(&sm.k_empty[buf]), ((items >> 1) & 1u) ^ 1u, ab)) return;
    unsigned char* k_tile = k_tiles + buf * T::TILE;
    constexpr int kBatch = 8;                             // loads in flight
#pragma unroll 1
    for (int i0 = 0; i0 < 128 / kLines; i0 += kBatch) {
      Eight<T> eight[kBatch] = {};
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (walk.inside) eight[i].load(a.kv, (int64_t)walk.pool_at + first + (i0 + i) * kLines, chunk);
#pragma unroll
      for (int i = 0; i < kBatch; ++i) *reinterpret_cast<uint4*>(k_tile + tile_chunk(first + (i0 + i) * kLines, chunk)) = eight[i].widen();
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.k_full[buf]));
    ++items;
    int token = walk.token + own_token;
    const float* lse = a.lse + (int64_t)(s.row0 + token) * a.lse_stride_row + (int64_t)(walk.at.head * a.group + own_head) * a.lse_stride_head;
    const int64_t step = tokens * a.lse_stride_row;
    for (int j0 = 0; j0 < walk.tiles; j0 += kAhead) {
      float own[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        own[i] = own_token < tokens && token < s.n_new ? __ldg(lse) : INFINITY;    // columns without a row: nothing
        token += tokens;
        lse += step;
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (j0 + i >= walk.tiles) break;
        const uint32_t slot = done % T::STAGES;
        if (!mbar_wait_warp(smem_u32(&sm.q_empty[slot]), ((done / T::STAGES) & 1u) ^ 1u, ab)) return;
        sm.below[done % kBelow][thread] = -own[i] * kLog2e;
        if (own[i] == -INFINITY) sm.idle = 1;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.b_full[slot]));
        ++done;
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------- products
template <class T>
__device__ __forceinline__ void multiply(const WeighArgs& w, Smem& sm, uint32_t tmem, uint32_t k_tiles, uint32_t q_ring, int64_t w0, int64_t w1, const Abort& ab) {
  constexpr uint32_t idesc = instr_desc(128, 128, false);
  const uint64_t k_desc = smem_desc<128>(k_tiles), q_desc = smem_desc<128>(q_ring);
  const bool on = elect_one();
  Walk walk(w, sm, w0, w1);
  uint32_t done = 0, items = 0;
  while (walk.next(w)) {
    if (walk.tiles == 0) continue;
    const uint32_t buf = items & 1u;
    if (!mbar_wait_warp(smem_u32(&sm.k_full[buf]), (items >> 1) & 1u, ab)) break;
    ++items;
    bool fine = true;
    for (int j = 0; j < walk.tiles; ++j, ++done) {
      const uint32_t slot = done % T::STAGES, acc = done % kAccs;
      const uint32_t parity = (done / T::STAGES) & 1u;
      fine = mbar_wait_warp(smem_u32(&sm.q_full[slot]), parity, ab) && mbar_wait_warp(smem_u32(&sm.b_full[slot]), parity, ab) && mbar_wait_warp(smem_u32(&sm.acc_empty[acc]), ((done / kAccs) & 1u) ^ 1u, ab);
      if (!fine) break;
      tc_fence_after();
      if (on) {
#pragma unroll
        for (int i = 0; i < T::D / 16; ++i) {
          const uint32_t at = (uint32_t)((i >> 2) * (128 * 128 >> 4) + 2 * (i & 3));
          tc_mma<false, false>(tmem + 128 * acc, k_desc + buf * (T::TILE >> 4) + at, q_desc + slot * (T::TILE >> 4) + at, idesc, (uint32_t)(i != 0));
        }
        tc_commit(smem_u32(&sm.q_empty[slot]));
        tc_commit(smem_u32(&sm.acc_full[acc]));
        mbar_arrive(smem_u32(&sm.acc_full[acc]));         // hands on what this warp has seen: the rows' log-sum-exps
        if (j + 1 == walk.tiles) tc_commit(smem_u32(&sm.k_empty[buf]));
      }
      __syncwarp();
    }
    if (!fine) break;
  }
  if (on) tc_commit(smem_u32(&sm.mma_done));
  __syncwarp();
  mbar_wait_warp(smem_u32(&sm.mma_done), 0u, ab);
}

// ---------------------------------------------------------------------------------------------- weights
// A tile's weights of a key where that is seldom: some row of the CTA's saw no key, which adds nothing, or a key with an infinite element makes NaN of
// the zeros behind a tile's last whole token.  Both by selection, whatever the products are, as for rows before `from`, and from `last` on, of the
// tile.  A function of its own: beside the other code it cost that 4 to 9 %.  Either gives other tiles the same bits, so that it does not matter when
// a warp first sees the flag for the former.
__device__ __noinline__ float2 add_seldom(uint32_t z_at, const float* below, float f, int from, int last) {
  uint64_t part[2] = {0ull, 0ull};
#pragma unroll 1
  for (int c = 0; c < 128; c += 4) {
    uint32_t four[4];
    tmem_issue<4>(z_at + c, four);
    tmem_load_wait();
    tmem_ready<4>(four);
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float b = below[c + i];
      p[i] = fast_exp2(fmaf(__uint_as_float(four[i]), f, b));
      if (c + i < from || c + i >= last || b == INFINITY) p[i] = 0.f;
    }
    part[0] = add2(part[0], pack2(p[0], p[1]));
    part[1] = add2(part[1], pack2(p[2], p[3]));
  }
  float2 both;
  unpack2(add2(part[0], part[1]), both.x, both.y);
  return both;
}

template <class T>
__device__ __forceinline__ void add_up(const WeighArgs& w, Smem& sm, uint32_t tmem, int64_t w0, int64_t w1, const Abort& ab) {
  const AttendArgs& a = w.a;
  const int lane = threadIdx.x & 31, set = (int)threadIdx.x >> 7, in = threadIdx.x & 127;
  const uint32_t lanes = (uint32_t)(in & ~31) << 16;
  const int64_t pool_rows = a.kv.n_blocks * a.kv.n_kv_heads * a.kv.block_tokens;
  Walk walk(w, sm, w0, w1);
  uint32_t done = 0, items = 0;                           // tiles before this item, items
  while (walk.next(w)) {
    const SeqSpan& s = walk.span.rows;
    const int tile_rows = tile_tokens(w) * a.group, row_first = walk.token * a.group, rows = s.n_new * a.group;
    const int key = walk.key0 + in;
    const bool books = set == 0 && walk.inside && key < s.end;
    float held = 0.f;
    if (books && key < walk.span.fresh) held = w.weight[(int64_t)walk.pool_at + in];
    int from = INT_MIN;                                   // the first row that sees the key
    if (key < s.first || key >= s.end) from = INT_MAX;
    else if (a.causal) from = (int)max(min(((int64_t)key - s.pos0) * a.group, (int64_t)INT_MAX), (int64_t)INT_MIN);
    float f = a.c;
    if constexpr (T::BITS == 8) f = logit_factor(a.c * group_scale(a.kv.k_scale, s, key & ~(kScaleTokens - 1), (walk.pool_at + in) & ~(kScaleTokens - 1), pool_rows), 1.f);
    const uint64_t ff = pack2(f, f);
    float sum = 0.f, lost = 0.f;
    for (int j = (int)(((uint32_t)set - done) % kSets); j < walk.tiles; j += kSets) {
      const uint32_t tile = done + (uint32_t)j, acc = tile % kAccs;
      if (!mbar_wait_warp(smem_u32(&sm.acc_full[acc]), (tile / kAccs) & 1u, ab)) return;
      tc_fence_after();
      const float* below = sm.below[tile % kBelow];
      const int rr = row_first + j * tile_rows;
      const int last = min(rows, rr + tile_rows);
      uint64_t part[2] = {0ull, 0ull};
      uint32_t z[2][16];
      tmem_issue<16>(tmem + 128 * acc + lanes, z[0]);
      // Of a key with an infinite element the zeros behind a tile's last whole token make NaN, as its last column shows.  (8- and 4-bit elements are
      // finite or NaN, and of NaN the rows that see the key make NaN too.)
      bool seldom = *const_cast<const volatile int*>(&sm.idle) != 0;
      if (T::BITS == 16 && tile_rows < 128) {
        uint32_t end[2];
        tmem_issue<2>(tmem + 128 * acc + lanes + 126, end);
        tmem_load_wait();
        tmem_ready<2>(end);
        seldom = seldom || __uint_as_float(end[1]) != __uint_as_float(end[1]);
      }
      // rows that do not see the key, and those behind the sequence's, which are other ones'
      const bool guard = __any_sync(0xffffffffu, rr < from || seldom) || rr + 128 > rows;
      if (guard && __any_sync(0xffffffffu, seldom)) {
        tmem_load_wait();
        tmem_ready<16>(z[0]);
        const float2 both = add_seldom(tmem + 128 * acc + lanes, below, f, max(from, 0) - rr, last - rr);
        part[0] = pack2(both.x, both.y);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.acc_empty[acc]));
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          tmem_load_wait();
          tmem_ready<16>(z[c & 1]);
          if (c < 7) {
            tmem_issue<16>(tmem + 128 * acc + lanes + 16 * (c + 1), z[(c + 1) & 1]);
          } else {
            tc_fence_before();                              // the accumulator is in registers
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.acc_empty[acc]));
          }
          float p[16];
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const float4 b = *reinterpret_cast<const float4*>(below + 16 * c + i);
            unpack2(fma2(pack2(z[c & 1][i], z[c & 1][i + 1]), ff, pack2(b.x, b.y)), p[i], p[i + 1]);
            unpack2(fma2(pack2(z[c & 1][i + 2], z[c & 1][i + 3]), ff, pack2(b.z, b.w)), p[i + 2], p[i + 3]);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) p[i] = fast_exp2(p[i]);
          if (guard) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (rr + 16 * c + i < from || rr + 16 * c + i >= last) p[i] = 0.f;
          }
#pragma unroll
          for (int i = 0; i < 16; i += 2) part[(i >> 1) & 1] = add2(part[(i >> 1) & 1], pack2(p[i], p[i + 1]));
        }
      }
      float u, v;
      unpack2(add2(part[0], part[1]), u, v);
      const float y = __fsub_rn(u + v, lost), t = __fadd_rn(sum, y);
      lost = __fsub_rn(__fsub_rn(t, sum), y);
      sum = t;
    }
    done += (uint32_t)walk.tiles;
    // the sets meet; the sums of two items lie apart
    float (&others)[kSets - 1][kKeys] = sm.sums[items & 1u];
    if (set > 0) others[set - 1][in] = sum;
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.summed));
    if (!mbar_wait_warp(smem_u32(&sm.summed), items & 1u, ab)) return;
    ++items;
    if (books) {
#pragma unroll
      for (int i = 0; i < kSets - 1; ++i) sum += others[i][in];
      book(w, (int64_t)walk.pool_at + in, held, sum, key, walk.span.fresh, walk.span.fresh_row);
    }
  }
}

template <int D, int BITS>
__global__ void __launch_bounds__(kThreads, 1) weigh_prompt_kernel(const __grid_constant__ WeighArgs w) {
  using T = Traits<D, BITS>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* k_tiles = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  unsigned char* q_ring = k_tiles + 2 * T::TILE;
  Smem& sm = *reinterpret_cast<Smem*>(q_ring + T::STAGES * T::TILE);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < T::STAGES; ++i) {
      mbar_init(smem_u32(&sm.q_full[i]), 1);
      mbar_init(smem_u32(&sm.q_empty[i]), 1);
      mbar_init(smem_u32(&sm.b_full[i]), 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sm.k_full[i]), 4);
      mbar_init(smem_u32(&sm.k_empty[i]), 1);
    }
    for (int i = 0; i < kAccs; ++i) {
      mbar_init(smem_u32(&sm.acc_full[i]), 2);
      mbar_init(smem_u32(&sm.acc_empty[i]), 4);
    }
    mbar_init(smem_u32(&sm.summed), 4 * kSets);
    mbar_init(smem_u32(&sm.mma_done), 1);
    sm.abort = 0;
    sm.idle = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 4 * kSets + 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // what the copies leave of a tile: rows of zeros
  for (int i = (tile_tokens(w) * w.a.group * 8) + (int)threadIdx.x; i < 128 * 8; i += kThreads)
    for (int t = 0; t < T::STAGES * (D / 64); ++t) reinterpret_cast<uint4*>(q_ring + t * (128 * 128))[i] = make_uint4(0u, 0u, 0u, 0u);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  find_start(w, sm);                                      // barriers of the CTA
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const int64_t per = (sm.total + gridDim.x - 1) / gridDim.x, w0 = per * blockIdx.x, w1 = min(w0 + per, sm.total);
  const Abort ab{&sm.abort, w.a.dev_status};
  if (w0 < w1) {
    if (warp < 4 * kSets) add_up<T>(w, sm, tmem, w0, w1, ab);
    else if (warp < 4 * kSets + 4) bring<T>(w, sm, k_tiles, w0, w1, ab);
    else if (warp == 4 * kSets + 5) copy_rows<T>(w, sm, smem_u32(q_ring), w0, w1, ab);
    else multiply<T>(w, sm, tmem, smem_u32(k_tiles), smem_u32(q_ring), w0, w1, ab);
  }
  tc_fence_before();
  __syncthreads();
  if (sm.abort != 0) {
    // a wait ran out: what is still in flight gets time to land before the memory is given back
    const unsigned long long t0 = global_timer();
    while (global_timer() - t0 < 2000000ull) __nanosleep(1000);
  }
  __syncthreads();
  if (warp == 4 * kSets + 4) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int D, int BITS>
int32_t launch(const WeighArgs& w, int sm_count, cudaStream_t stream) {
  constexpr int kBytes = smem_bytes<Traits<D, BITS>>();
  static_assert(kBytes <= 227 * 1024);
  static ContextSet done;
  const int32_t st = allow_shared_memory(reinterpret_cast<const void*>(weigh_prompt_kernel<D, BITS>), kBytes, done);
  if (st != SPF_OK) return st;
  weigh_prompt_kernel<D, BITS><<<sm_count, kThreads, kBytes, stream>>>(w);
  SPF_CUDA_CHECK(cudaGetLastError());
  return SPF_OK;
}

}  // namespace

// Strides of zero, which a row or a head for all has, and of 2^40 bytes and more are not a tensor map's; neither are more than 128 heads to a
// key head a tile's.
bool weigh_prompt_prepare(WeighArgs& w, int n_q_heads, int head_dim) {
  const RowsView& q = w.a.q;
  const int64_t most = (int64_t)1 << 38;
  if (w.a.group > 128 || q.stride_row <= 0 || q.stride_head <= 0 || q.stride_row >= most || q.stride_head >= most) return false;
  const bool fine = encode_rows_map("spf_kv_weigh", q, w.a.step.n_rows, n_q_heads, head_dim, 128 / w.a.group, w.a.group, &w.q_map) == SPF_OK;
  if (!fine) clear_error();                               // the other kernel takes them
  return fine;
}

int32_t weigh_prompt_launch(const WeighArgs& w, int head_dim, int sm_count, cudaStream_t stream) {
  const bool d64 = head_dim == 64;
  switch (w.a.kv.bits) {
    case 4: return d64 ? launch<64, 4>(w, sm_count, stream) : launch<128, 4>(w, sm_count, stream);
    case 8: return d64 ? launch<64, 8>(w, sm_count, stream) : launch<128, 8>(w, sm_count, stream);
    default: return d64 ? launch<64, 16>(w, sm_count, stream) : launch<128, 16>(w, sm_count, stream);
  }
}

}  // namespace spf
