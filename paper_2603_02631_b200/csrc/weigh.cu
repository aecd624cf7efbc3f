// The attention weights that the cache's tokens receive from a step's rows, added to the ledger beside the cache.
//
//   W[h, s] = decay W[h, s] + sum over rows r that see s of 2^(z[r,s] - lse2[r]),   z[r,s] = c q[r] . k[s],   rows r = (new token, head of h's group)
//
// One pass over the keys: a row's log-sum-exp is known (its attention came first), so a weight is final as soon as its logit is there, and tiles
// of keys are independent of one another.  The work is the list of all key tiles of all (sequence, key head), cut into one part for each CTA.
// Copies, products and the 4-bit keys' arithmetic are those of the attention for few rows (8-bit keys are multiplied in bf16 here); a thread's weights of a key are summed
// over its rows, the four lanes that share a key exchange sums, and each of them books one key.  With more rows than a tile of R the tile of keys
// stays where it is while the rows go by, up to 128 of them from shared memory.
//
// What bounds it with few rows is the read of the keys, of which it misses half: one token for each of 32 sequences of up to 16k tokens on a 4-bit
// cache, 8 heads of 128 dimensions, takes 52 us where the bytes take 27; without any product it takes 46, with 8 us of launch and first loads.
// (Where it took 58 it took 61 with the ledger's weights loaded when they are wanted, not copied with the keys.)
// Masks stand apart from the exponentials, in a block of their own: as a condition on each they made a branch of each (95 instead of
// 36 us for 128 rows over 32k keys of 64 dimensions, 33 now, whose exponentials take 8).
#include <algorithm>
#include <cmath>

#include "attend_step.cuh"
#include "weigh.cuh"

namespace spf {
namespace {

// Tiles of rows whose weights are added up plainly: up to 128 rows, for which the kernel is meant, have four.  With more (a hint that is too small,
// rows that the other kernel does not take) sums carry what each addition loses, in a kernel of its own (MANY): there are no registers to spare for it
// (a token of 32 sequences, 4 bits, 52.6 us instead of 51.2).
constexpr int kPlain = 8;

// What the copying warp tells the computing ones about a stage.
struct WeighDesc {
  int row0, n_new, pos0, first, end, head, key0, fresh, fresh_row;
  int cell;                             // of the first key in the ledger, below zero: the block lies outside the pool
  float k_scale[2];                     // 8 bits: of the tile's groups of 64 keys
  int new_rows;                         // the stage's rows are not those of the stage before
};

template <class T>
struct WeighSmem {
  float held[T::STAGES][T::KEYS];       // what the ledger holds of the stages' keys
  unsigned long long full[kMaxStages], empty[kMaxStages], join;
  WeighDesc desc[kMaxStages];
  int64_t scan[kWarps + 1];
  int64_t total, start_base;
  int start_seq;
  int abort;
};

template <class T>
constexpr int weigh_smem_bytes() { return T::STAGES * T::STAGE + T::TILES_HELD * T::QBYTES + (int)sizeof(WeighSmem<T>) + 1024; }

// Tiles of a (sequence, key head): all keys, since what no row sees is still multiplied by the decay.
template <class T>
__device__ __forceinline__ int weigh_tiles(const SeqSpan& s) { return (s.end + T::KEYS - 1) / T::KEYS; }
template <class T>
__device__ __forceinline__ int64_t weigh_cost(const WeighArgs& w, int b) {
  const SeqSpan s = seq_span(w.a, b);
  return s.n_new > 0 ? (int64_t)w.a.kv.n_kv_heads * weigh_tiles<T>(s) : 0;
}

// Length of the list, and the sequence that holds the CTA's first tile.
template <class T>
__device__ __forceinline__ void weigh_start(const WeighArgs& w, WeighSmem<T>& sm) {
  const int n_seqs = w.a.step.n_seqs, run = (n_seqs + T::THREADS - 1) / T::THREADS, lo = min((int)threadIdx.x * run, n_seqs), hi = min(lo + run, n_seqs);
  int64_t mine = 0;
  for (int b = lo; b < hi; ++b) mine += weigh_cost<T>(w, b);
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
#pragma unroll
  for (int i = 0; i < T::THREADS / 32; ++i) {
    if (i < warp) upto += sm.scan[i];
    total += sm.scan[i];
  }
  const int64_t w0 = (total + gridDim.x - 1) / gridDim.x * blockIdx.x;
  if (threadIdx.x == 0) sm.total = total;
  if (w0 >= upto - mine && w0 < upto) {
    int64_t base = upto - mine;
    int b = lo;
    for (; b < hi - 1; ++b) {
      const int64_t c = weigh_cost<T>(w, b);
      if (w0 < base + c) break;
      base += c;
    }
    sm.start_seq = b;
    sm.start_base = base;
  }
  __syncthreads();
}

template <class T>
__device__ __forceinline__ void copy_keys(const WeighArgs& w, WeighSmem<T>& sm, uint32_t ring, int64_t w0, int64_t w1, const Abort& ab) {
  const AttendArgs& a = w.a;
  const int lane = threadIdx.x & 31;
  const int64_t pool_rows = a.kv.n_blocks * a.kv.n_kv_heads * a.kv.block_tokens;
  int seq = sm.start_seq;
  int64_t base = sm.start_base;
  int stage = 0;
  int64_t issued = 0;
  uint32_t parity = 1;                                    // the ring's stages start out empty
  for (int64_t at = w0; at < w1; at += 32) {
    // each lane works out one of the next 32 tiles
    const int64_t mine = at + lane;
    WeighDesc d{};
    int row = 0;
    if (mine < w1) {
      int64_t cost = weigh_cost<T>(w, seq);
      while (mine >= base + cost && seq < a.step.n_seqs - 1) {
        base += cost;
        cost = weigh_cost<T>(w, ++seq);
      }
      const WeighSpan s = weigh_span(w, seq);
      const int tiles = weigh_tiles<T>(s.rows);
      const int64_t in_seq = mine - base;
      d.row0 = s.rows.row0, d.n_new = s.rows.n_new, d.pos0 = s.rows.pos0, d.first = s.rows.first, d.end = s.rows.end;
      d.fresh = s.fresh, d.fresh_row = s.fresh_row;
      d.head = (int)(in_seq / tiles);
      const int tile = (int)(in_seq - (int64_t)d.head * tiles);
      d.key0 = tile * T::KEYS;
      d.new_rows = mine == w0 || tile == 0;
      row = pool_row(a, seq, d.head, d.key0);
      d.cell = row < pool_rows ? row : -1;
      if constexpr (T::FP8) {
#pragma unroll
        for (int g = 0; g < T::KEYS / kScaleTokens; ++g)
          d.k_scale[g] = a.c * group_scale(a.kv.k_scale, s.rows, d.key0 + g * kScaleTokens, row + g * kScaleTokens, pool_rows);
      }
    }
    const int count = (int)min((int64_t)32, w1 - at);
    for (int j = 0; j < count; ++j) {
      if (!mbar_wait_warp(smem_u32(&sm.empty[stage]), parity, ab)) {
        if (lane < T::STAGES && issued > lane)
          drain_copy(smem_u32(&sm.full[lane]), (uint32_t)((issued - lane + T::STAGES - 1) / T::STAGES - 1) & 1u);
        return;
      }
      ++issued;
      if (lane == j) {
        sm.desc[stage] = d;
        const uint32_t bar = smem_u32(&sm.full[stage]), to = ring + stage * T::STAGE;
        mbar_expect_tx(bar, T::STAGE + T::KEYS * 4);
        tma_load_3d(to, &w.k_map, 0, row, 0, bar);
        tma_load_2d(smem_u32(sm.held[stage]), &w.weight_map, 0, row / T::KEYS, bar);
        if constexpr (T::INT4) tma_load_2d(to + T::TILE, &w.k_scale_map, 0, row / 128, bar);
      }
      if (++stage == T::STAGES) stage = 0, parity ^= 1;
    }
    seq = __shfl_sync(0xffffffffu, seq, count - 1);
    base = __shfl_sync(0xffffffffu, base, count - 1);
  }
}

// Base-2 log-sum-exp of the row `row` of `total` that a sequence has for a key head, -inf for one that saw no key, whose weights are set to zero.
// A tile is filled up with copies of the last row (load_queries), which sees every key that any row does, and the largest number as their
// log-sum-exp: a copy adds 0, or the infinity or NaN that the row itself adds.  (Zeros in their place make NaN of a key with an infinite element.)
__device__ __forceinline__ float row_lse2(const AttendArgs& a, const WeighDesc& d, int row, int total) {
  const int r = min(row, total - 1);
  const float lse = __ldg(a.lse + (int64_t)(d.row0 + r / a.group) * a.lse_stride_row + (int64_t)(d.head * a.group + r % a.group) * a.lse_stride_head);
  return row < total || lse == -INFINITY ? lse * kLog2e : 3.402823466e38f;
}

template <class T, bool MANY>
__device__ __forceinline__ void weigh_tiles_of_cta(const WeighArgs& w, WeighSmem<T>& sm, uint32_t ring, unsigned char* q_tile, int64_t n_tiles, const Abort& ab) {
  constexpr int R = T::R, NT = T::NT, KT = T::KT;
  static_assert(T::WR == 1 && KT <= 2);
  const AttendArgs& a = w.a;
  const int lane = threadIdx.x & 31, key_off = (threadIdx.x >> 5) * T::KW;
  const uint32_t q_addr = smem_u32(q_tile);
  constexpr int kHeld = T::TILES_HELD;
  __shared__ QueryNotes<T> notes[kHeld];
  __shared__ float lse2[kHeld][R];
  Queries<T> queries;
  float below[NT][2];                                    // the rows' log-sum-exps
  uint32_t idle = 0;                                     // tiles of rows, of those held, with some that saw no key
  int first_token = 0, last_token = 0;                   // of the rows of the tile
  int stage = 0;
  uint32_t parity = 0, join_parity = 0;
  auto join = [&] {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.join));
    const bool ok = mbar_wait_warp(smem_u32(&sm.join), join_parity, ab);
    join_parity ^= 1;
    return ok;
  };
  // the key that a thread books: lane % 4 = 2 kt + half
  const int own = key_off + (KT == 2 ? ((lane >> 1) & 1) * 16 : 0) + key_of<T>(lane, lane & 1);
  const bool books = KT == 2 || (lane & 3) < 2;
  for (int64_t tile = 0; tile < n_tiles; ++tile) {
    if (!mbar_wait_warp(smem_u32(&sm.full[stage]), parity, ab)) return;
    const WeighDesc& d = sm.desc[stage];
    const int key0 = d.key0, end = d.end, first = d.first, own_key = key0 + own;
    const bool writes = books && d.cell >= 0 && own_key < end;
    const int64_t cell = (int64_t)d.cell + own;
    const int row_tiles = (int)(((int64_t)d.n_new * a.group + R - 1) / R);
    float got[KT][2] = {}, lost[MANY ? KT : 1][2] = {};   // sums over tiles of rows, and what their additions lose
    for (int rt = 0; rt < row_tiles; ++rt) {
      const int slot = rt % kHeld;
      if (slot == 0 && (d.new_rows || row_tiles > kHeld)) {
        // the warps are through with the rows before these, then they have all brought these
        if (tile > 0 || rt > 0) {
          if (!join()) return;
        }
        for (int i = 0; i < min(kHeld, row_tiles - rt); ++i) {
          TileDesc t;
          t.row0 = d.row0, t.n_new = d.n_new, t.head = d.head, t.row_tile = rt + i;
          load_queries<T>(a, t, q_tile + i * T::QBYTES, notes[i]);
          for (int r = threadIdx.x; r < R; r += kWarps * 32) lse2[i][r] = row_lse2(a, d, (rt + i) * R + r, d.n_new * a.group);
        }
        if (!join()) return;
        idle = 0;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) idle |= __any_sync(0xffffffffu, lse2[i][lane % R] == -INFINITY) ? 1u << i : 0u;
      }
      if (d.new_rows || row_tiles > 1) {
        queries.load(q_addr + slot * T::QBYTES, notes[slot], 0, lane);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) below[nt][e] = lse2[slot][nt * 8 + 2 * (lane & 3) + e];
        first_token = rt * R / a.group, last_token = min(d.n_new - 1, (rt * R + R - 1) / a.group);
      }
      const int row_first = rt * R, seen_by_all = a.causal ? min(end, d.pos0 + first_token + 1) : end;
      if (a.causal && d.pos0 + last_token < key0) continue;    // no row of the tile sees any of these keys
      const bool guard = key0 < first || key0 + T::KEYS > seen_by_all;
      const uint32_t k_tile = ring + stage * T::STAGE;
      const float k_scale = T::FP8 ? d.k_scale[T::KEYS > kScaleTokens ? key_off / kScaleTokens : 0] : a.c;
      float z[KT][NT][4];
      tile_logits<T>(z, queries, q_addr + slot * T::QBYTES, 0, k_tile, k_tile + T::TILE, key_off, lane);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) f[e] = T::FP8 ? logit_factor(k_scale, queries.factor[nt][e]) : T::INT4 ? queries.factor[nt][e] : k_scale;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[kt][nt][e] = fast_exp2(fmaf(z[kt][nt][e], f[e & 1], -below[nt][e & 1]));
      }
      if ((idle >> slot & 1u) != 0) {
        // by selection, whatever their products are
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) z[kt][nt][e] = below[nt][e & 1] == -INFINITY ? 0.f : z[kt][nt][e];
      }
      if (guard) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            // rows from (key - pos0) group on see a key
            const int key = key0 + key_off + kt * 16 + key_of<T>(lane, h);
            const int64_t from = key < first || key >= end ? INT64_MAX : a.causal ? ((int64_t)key - d.pos0) * a.group : 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (row_first + nt * 8 + 2 * (lane & 3) + e < from) z[kt][nt][2 * h + e] = 0.f;
          }
      }
      float part[KT][2] = {};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int h = 0; h < 2; ++h) (MANY ? part : got)[kt][h] += z[kt][nt][2 * h] + z[kt][nt][2 * h + 1];
      if constexpr (MANY) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float y = __fsub_rn(part[kt][h], lost[kt][h]), t = __fadd_rn(got[kt][h], y);
            lost[kt][h] = __fsub_rn(__fsub_rn(t, got[kt][h]), y);
            got[kt][h] = t;
          }
      }
    }
    // sums over the four lanes of a key, each of which ends with one key's
    float sum;
    if constexpr (KT == 2) {
      const bool up = (lane & 2) != 0, odd = (lane & 1) != 0;
      const float s0 = (up ? got[1][0] : got[0][0]) + __shfl_xor_sync(0xffffffffu, up ? got[0][0] : got[1][0], 2);
      const float s1 = (up ? got[1][1] : got[0][1]) + __shfl_xor_sync(0xffffffffu, up ? got[0][1] : got[1][1], 2);
      sum = (odd ? s1 : s0) + __shfl_xor_sync(0xffffffffu, odd ? s0 : s1, 1);
    } else {
      const bool odd = (lane & 1) != 0;
      sum = (odd ? got[0][1] : got[0][0]) + __shfl_xor_sync(0xffffffffu, odd ? got[0][0] : got[0][1], 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    }
    if (writes) book(w, cell, sm.held[stage][own], sum, own_key, d.fresh, d.fresh_row);
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.empty[stage]));
    if (++stage == T::STAGES) stage = 0, parity ^= 1;
  }
}

template <class T, bool MANY>
__global__ void __launch_bounds__(T::THREADS, T::CTAS) weigh_step_kernel(const __grid_constant__ WeighArgs w) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring_ptr = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  unsigned char* q_tile = ring_ptr + T::STAGES * T::STAGE;
  WeighSmem<T>& sm = *reinterpret_cast<WeighSmem<T>*>(q_tile + T::TILES_HELD * T::QBYTES);
  if (threadIdx.x == 0) {
    for (int i = 0; i < T::STAGES; ++i) {
      mbar_init(smem_u32(&sm.full[i]), 1);
      mbar_init(smem_u32(&sm.empty[i]), kWarps);
    }
    mbar_init(smem_u32(&sm.join), kWarps);
    sm.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  weigh_start<T>(w, sm);                                 // ends with a barrier of the CTA
  const int64_t total = sm.total, per = (total + gridDim.x - 1) / gridDim.x, w0 = per * blockIdx.x, w1 = min(w0 + per, total);
  if (w0 >= w1) return;
  const Abort ab{&sm.abort, w.a.dev_status};
  if (threadIdx.x < kWarps * 32) weigh_tiles_of_cta<T, MANY>(w, sm, smem_u32(ring_ptr), q_tile, w1 - w0, ab);
  else copy_keys<T>(w, sm, smem_u32(ring_ptr), w0, w1, ab);
}

template <class T, bool MANY>
int32_t launch_kernel(const WeighArgs& w, int sm_count, cudaStream_t stream) {
  static ContextSet done;
  const int32_t st = allow_shared_memory(reinterpret_cast<const void*>(weigh_step_kernel<T, MANY>), weigh_smem_bytes<T>(), done);
  if (st != SPF_OK) return st;
  weigh_step_kernel<T, MANY><<<sm_count * T::CTAS, T::THREADS, weigh_smem_bytes<T>(), stream>>>(w);
  SPF_CUDA_CHECK(cudaGetLastError());
  return SPF_OK;
}
// `most`: rows that a key head and sequence may have.
template <int D, int BITS, int R>
int32_t launch_weigh(WeighArgs& w, const spf_kv_cache* cache, int64_t most, int sm_count, cudaStream_t stream) {
  using T = Traits<D, BITS, R, false>;
  int32_t st = encode_pool_map("spf_kv_weigh", cache, cache->k_pool, T::KEYS, &w.k_map);
  if (st == SPF_OK) st = encode_ledger_map("spf_kv_weigh", cache, w.weight, T::KEYS, &w.weight_map);
  if constexpr (T::INT4) {
    if (st == SPF_OK) st = encode_scale_map("spf_kv_weigh", cache, cache->k_scale, &w.k_scale_map);
  }
  if (st != SPF_OK) return st;
  return most > kPlain * R ? launch_kernel<T, true>(w, sm_count, stream) : launch_kernel<T, false>(w, sm_count, stream);
}
template <int D, int BITS>
int32_t launch_rows(WeighArgs& w, const spf_kv_cache* cache, int64_t rows, int64_t most, int sm_count, cudaStream_t stream) {
  if (rows <= 8) return launch_weigh<D, BITS, 8>(w, cache, most, sm_count, stream);
  if (rows <= 16) return launch_weigh<D, BITS, 16>(w, cache, most, sm_count, stream);
  return launch_weigh<D, BITS, 32>(w, cache, most, sm_count, stream);
}

}  // namespace
}  // namespace spf

using namespace spf;

extern "C" int32_t spf_kv_weigh(const spf_kv_cache* cache, const spf_kv_step* step, const spf_rows* q, int32_t n_q_heads, float softmax_scale,
                                const spf_attend_options* attend, const spf_kv_ledger* ledger, const spf_kv_weigh_options* options,
                                int32_t* dev_status, void* cuda_stream) {
  const char* who = "spf_kv_weigh";
  clear_error();
  WeighArgs w{};
  AttendArgs& a = w.a;
  int32_t st = check_cache(who, cache, &a.kv);
  if (st == SPF_OK) st = check_step(who, step, &a.step);
  if (st == SPF_OK) st = check_heads(who, cache, n_q_heads, &a.group);
  if (st == SPF_OK) st = check_ledger(who, ledger);
  if (st != SPF_OK) return st;
  w.weight = ledger->weight;
  w.position = ledger->position;
  w.decay = 1.f;
  if (options != nullptr) {
    if (!(options->decay >= 0.f) || !std::isfinite(options->decay)) return fail(SPF_ERR_INVALID_ARG, "%s: decay must be finite and not negative", who);
    if (options->last_rows < 0) return fail(SPF_ERR_INVALID_ARG, "%s: last_rows must not be negative", who);
    w.decay = options->decay;
    w.last_rows = options->last_rows;
    w.positions = options->positions;
  }
  if (step->n_rows == 0) return SPF_OK;
  if (attend == nullptr || attend->lse == nullptr) return fail(SPF_ERR_INVALID_ARG, "%s: lse is null", who);
  st = check_rows(who, "q", q, n_q_heads, cache->head_dim, false, &a.q);
  if (st == SPF_OK) st = attend_settings(who, cache, step, n_q_heads, softmax_scale, attend, &a);
  if (st != SPF_OK) return st;
  a.dev_status = dev_status;
  int sm_count = 0;
  st = device_sm_count(&sm_count);
  if (st != SPF_OK) return st;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  auto rows_of = [&](int64_t tokens) { return a.group * (w.last_rows > 0 ? std::min<int64_t>(w.last_rows, tokens) : tokens); };
  const int64_t rows = rows_of(step->max_new);
  // Rows that the sequences cannot have by the hint: then some may have all of them.  (Fewer, in one sequence, may be more than it says too: not more
  // than the hint allows all sequences together.)
  const int64_t most = step->n_rows > (int64_t)step->n_seqs * step->max_new ? std::max(rows, rows_of(step->n_rows)) : rows;
  // Both over 131072 keys and over 8 sequences of 4000, 8 key heads, first against second kernel.  128 rows: bf16 95 against 174 us and 34 against 48
  // (64 dimensions), 154 against 201 and 52 against 54 (128); 8 bits 121 against 225, 43 against 57 and 184 against 252, 63 against 66; 4 bits 126
  // against 197, 46 against 52, but 254 against 213, 86 against 61 with 128 dimensions, whose codes are unpacked for each 32 rows anew (64 rows:
  // 139 against 248, 48 against 69).  256 rows: 304 against 189 (bf16, 64 dimensions) to 819 against 226 (4 bits, 128).
  const int64_t few = a.kv.bits == 4 && cache->head_dim == 128 ? 64 : 128;
  if (rows > few && weigh_prompt_prepare(w, n_q_heads, cache->head_dim)) return weigh_prompt_launch(w, cache->head_dim, sm_count, stream);
  const bool d64 = cache->head_dim == 64;
  switch (a.kv.bits) {
    case 4: return d64 ? launch_rows<64, 4>(w, cache, rows, most, sm_count, stream) : launch_rows<128, 4>(w, cache, rows, most, sm_count, stream);
    case 8: return d64 ? launch_rows<64, 8>(w, cache, rows, most, sm_count, stream) : launch_rows<128, 8>(w, cache, rows, most, sm_count, stream);
    default: return d64 ? launch_rows<64, 16>(w, cache, rows, most, sm_count, stream) : launch_rows<128, 16>(w, cache, rows, most, sm_count, stream);
  }
}
