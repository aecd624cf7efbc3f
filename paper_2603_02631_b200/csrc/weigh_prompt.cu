// The attention weights that the cache's tokens receive from a step with many rows per key head (chunks of prompts).
//
//   W[h, s] = decay W[h, s] + sum over rows r that see s of 2^(f_s q[r] . k[s] - lse2[r])
//
// Here the exponentials bound it (128 rows by 128 keys take the exponential unit 1024 cycles, the warp-level products of 128 dimensions as
// long, the big instruction's a quarter), so a weight should cost little else.  A CTA has 128 keys of a (sequence, key head) in registers, as
// left operands of warp-level products, widened to bf16 once (exactly: 8-bit values, and 4-bit codes times scales of five bits), and the
// rows go by in stages of 128.  A warp has 32 keys and every fourth 32 rows: logits have keys as rows and query rows as columns, so a thread's
// weights of a key add up in registers, and only at the end do the lanes and warps that share a key exchange sums.  Sums of a stage are
// added with what the additions lose (thousands of rows make 1.7e-6 of a weight otherwise).
//
// The list of all (sequence, key head, 128 keys), each as long as the stages of rows that see any of its keys, is cut into one part for each SM; an
// item belongs to the part that its beginning lies in.
#include <climits>

#include "weigh.cuh"

namespace spf {
namespace {

constexpr int kThreads = 512, kKeys = 128, kStages = 3, kKeyGroups = 4, kRowGroups = 4;
constexpr int kGroupRows = 64, kRows = kRowGroups * kGroupRows, kGroupThreads = kThreads / kRowGroups;

template <int D_, int BITS_>
struct Traits {
  static constexpr int D = D_, BITS = BITS_, BLOCKS = D / 32, QSTAGE = kGroupRows * D * 2;
  static constexpr int STEP = D == 64 ? 2 : 1;            // eights of rows whose products are under way together
};

struct Smem {
  float below[kRowGroups][kStages][kGroupRows];           // the rows' base-2 log-sum-exps, negated
  float sums[kRowGroups][kKeys];
  int64_t scan[kThreads / 32];
  int64_t total, start_base;
  int start_seq;
};

// ---------------------------------------------------------------------------------------------- the list of items
// Rows of a sequence and key head, from the first that sees key0 on (a multiple of 8).
__device__ __forceinline__ int first_row(const WeighArgs& w, const SeqSpan& s, int key0) {
  if (!w.a.causal) return 0;
  const int64_t r = ((int64_t)key0 - s.pos0) * w.a.group;
  return (int)min(max(r, (int64_t)0), (int64_t)s.n_new * w.a.group) & ~7;
}
__device__ __forceinline__ int stages_of(const WeighArgs& w, const SeqSpan& s, int key0) {
  if (key0 + kKeys <= s.first) return 0;
  return (int)(((int64_t)s.n_new * w.a.group - first_row(w, s, key0) + kRows - 1) / kRows);
}
// Length of a (sequence, key head) in the list: its stages, and one more an item for its beginning and end.
__device__ __forceinline__ int64_t head_cost(const WeighArgs& w, const SeqSpan& s) {
  const int tiles = (s.end + kKeys - 1) / kKeys;
  // keys before the first that every row sees, and those from the first row's on
  const int before = s.first / kKeys, all = w.a.causal ? min(max(s.pos0, 0) / kKeys, tiles) : tiles;
  int64_t cost = tiles;
  if (all > before) cost += (int64_t)(all - before) * stages_of(w, s, before * kKeys);
  for (int t = max(all, before); t < tiles; ++t) cost += stages_of(w, s, t * kKeys);
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
  if (all > before && w0 > c.at + before) {
    // among the items of equal length, without looking at each
    const int64_t each = stages_of(w, s, before * kKeys) + 1, skip = min((w0 - c.at - before) / each, (int64_t)(all - before));
    c.tile = before + (int)skip;
    c.at += before + skip * each;
  }
  while (c.at < w0) c.at += stages_of(w, s, c.tile++ * kKeys) + 1;
  return c;
}

// ---------------------------------------------------------------------------------------------- keys
__device__ __forceinline__ uint32_t mul_bf16(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Eight elements of a key from dimension 8 j on as bf16 pairs; `row` is the key's row in the pool.
template <class T>
__device__ __forceinline__ void load_eight(const KvView& kv, int64_t row, int j, uint32_t (&r)[4]) {
  if constexpr (T::BITS == 16) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(kv.k + row * (2 * T::D)) + j);
    r[0] = v.x, r[1] = v.y, r[2] = v.z, r[3] = v.w;
  } else if constexpr (T::BITS == 8) {
    const uint2 v = __ldg(reinterpret_cast<const uint2*>(kv.k + row * T::D) + j);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t word = i < 2 ? v.x : v.y, two = __byte_perm(word, 0, i & 1 ? 0x4342 : 0x4140);
      // a byte s eeee mmm at the bits s 0000eeee mmm0000 is its value times 2^-120
      r[i] = mul_bf16(((two << 8) & 0x80008000u) | ((two << 4) & 0x07f007f0u), 0x7b807b80u);
      if ((((two & 0x007f007fu) + 0x00010001u) & 0x00800080u) != 0) {
        if ((two & 0x7fu) == 0x7fu) r[i] |= 0x00007fffu;
        if ((two & 0x7f0000u) == 0x7f0000u) r[i] |= 0x7fff0000u;
      }
    }
  } else {
    const uint32_t word = __ldg(reinterpret_cast<const uint32_t*>(kv.k + row * (T::D / 2)) + j);
    const uint32_t s = __ldg(kv.k_scale4 + row * T::BLOCKS + j / 4), both = s | s << 16, less = mul_bf16(both, 0xc1c0c1c0u);   // -24 scales
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = word >> (8 * i);
      r[i] = ((two & 0xfu) << 3) | ((two & 0xf0u) << 15) | 0x41804180u;                                                        // 16 + code
      asm("fma.rn.bf16x2 %0, %0, %1, %2;" : "+r"(r[i]) : "r"(both), "r"(less));
    }
  }
}

// ---------------------------------------------------------------------------------------------- rows
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same with nothing to add to.
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Byte offset of a row's 16-byte chunk in a stage: rows in turns begin with either half of 128 bytes, so that two rows' four chunks touch every bank.
template <class T>
__device__ __forceinline__ uint32_t row_chunk(int row, int chunk) { return (uint32_t)(row * (2 * T::D) + (chunk ^ ((row & 1) << 2)) * 16); }

// A row of a sequence and key head as (token, head of the group), and the step to one further on, without a division.
struct RowAt {
  int token, g;
  __device__ __forceinline__ RowAt(int64_t rr, int group) : token((int)(rr / group)), g((int)(rr - (int64_t)token * group)) {}
  __device__ __forceinline__ RowAt after(const RowAt& step, int group) const {
    RowAt r = *this;
    r.token += step.token, r.g += step.g;
    if (r.g >= group) r.g -= group, ++r.token;
    return r;
  }
};

// Asks for the rows of a stage, from (token, g) `at` on, the thread's first; `lse_at` is that of the thread's log-sum-exp, which is returned.
template <class T>
__device__ __forceinline__ float fetch_rows(const WeighArgs& w, const SeqSpan& s, int head, RowAt at, const RowAt& lse_at, const RowAt& step, uint32_t to) {
  constexpr int kChunks = T::D / 8;
  const AttendArgs& a = w.a;
  const int thread = (int)threadIdx.x % kGroupThreads, first = thread / kChunks, chunk = thread % kChunks;
  const __nv_bfloat16* base = a.q.data + s.row0 * a.q.stride_row + (int64_t)head * a.group * a.q.stride_head + 8 * chunk;
#pragma unroll
  for (int i = 0; i < kGroupRows * kChunks / kGroupThreads; ++i) {
    const int r = first + i * (kGroupThreads / kChunks), bytes = at.token < s.n_new ? 16 : 0;     // rows that do not exist are zeros
    const __nv_bfloat16* src = base + (bytes ? at.token * a.q.stride_row + at.g * a.q.stride_head : 0);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + row_chunk<T>(r, chunk)), "l"(src), "r"(bytes) : "memory");
    at = at.after(step, a.group);
  }
  return thread < kGroupRows ? row_lse2(a, s.row0 + lse_at.token, head * a.group + lse_at.g, lse_at.token < s.n_new) : 0.f;
}

template <int D, int BITS>
__global__ void __launch_bounds__(kThreads, 1) weigh_prompt_kernel(const __grid_constant__ WeighArgs w) {
  using T = Traits<D, BITS>;
  extern __shared__ __align__(128) unsigned char q_rows[];
  __shared__ Smem sm;
  const AttendArgs& a = w.a;
  find_start(w, sm);
  const int64_t per = (sm.total + gridDim.x - 1) / gridDim.x, w0 = per * blockIdx.x, w1 = min(w0 + per, sm.total);
  if (w0 >= w1) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, key_group = warp % kKeyGroups, row_group = warp / kKeyGroups, c = lane & 3;
  const int in_group = (int)threadIdx.x % kGroupThreads;
  const unsigned char* group_rows = q_rows + row_group * kStages * T::QSTAGE;
  const uint32_t q_addr = smem_u32(group_rows);           // of the copies
  const int64_t pool_rows = a.kv.n_blocks * a.kv.n_kv_heads * a.kv.block_tokens;
  const RowAt copy_step(kGroupThreads / (D / 8), a.group), stage_step(kRows, a.group);   // from a thread's row to its next, from a stage to the next
  Cursor cur = first_item(w, sm, w0);
  WeighSpan span = weigh_span(w, cur.seq);
  while (cur.at < w1) {
    // the next item: heads and sequences behind one another
    while (span.rows.n_new <= 0 || cur.tile * kKeys >= span.rows.end) {
      cur.tile = 0;
      if (span.rows.n_new <= 0 || span.rows.end == 0 || ++cur.head >= a.kv.n_kv_heads) {
        cur.head = 0;
        if (++cur.seq >= a.step.n_seqs) return;
        span = weigh_span(w, cur.seq);
      }
    }
    const SeqSpan& s = span.rows;
    const int key0 = cur.tile * kKeys, stages = stages_of(w, s, key0);
    const int row_first = first_row(w, s, key0);
    const int pool_at = pool_row(a, cur.seq, cur.head, key0);
    const bool inside = pool_at < pool_rows;
    float lse2[2];                                        // of the stages under way
    const int group_first = row_first + row_group * kGroupRows;
    RowAt copy_at(group_first + in_group / (D / 8), a.group), lse_at(group_first + in_group % kGroupRows, a.group);
    auto fetch = [&](int slot) {
      const float x = fetch_rows<T>(w, s, cur.head, copy_at, lse_at, copy_step, q_addr + slot * T::QSTAGE);
      copy_at = copy_at.after(stage_step, a.group), lse_at = lse_at.after(stage_step, a.group);
      return x;
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lse2[i] = i < stages ? fetch(i) : 0.f;
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    float held = 0.f;
    const int own = key0 + (int)threadIdx.x;
    const bool books = threadIdx.x < kKeys && inside && own < s.end;
    if (books && own < span.fresh) held = w.weight[(int64_t)pool_at + threadIdx.x];
    // the warp's keys
    uint32_t k[2][T::BLOCKS][2][4];
    int from[2][2];                                       // the first row that sees a key
    int guard_below = INT_MIN;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int in = key_group * 32 + kt * 16 + h * 8 + (lane >> 2), key = key0 + in;
#pragma unroll
        for (int b = 0; b < T::BLOCKS; ++b) {
          if (stages > 0 && inside) load_eight<T>(a.kv, (int64_t)pool_at + in, 4 * b + c, k[kt][b][h]);
          else k[kt][b][h][0] = k[kt][b][h][1] = k[kt][b][h][2] = k[kt][b][h][3] = 0u;
        }
        if (key < s.first || key >= s.end) from[kt][h] = INT_MAX;
        else from[kt][h] = a.causal ? (int)max(min(((int64_t)key - s.pos0) * a.group, (int64_t)INT_MAX), (int64_t)INT_MIN) : INT_MIN;
        guard_below = max(guard_below, from[kt][h]);
      }
    guard_below = __reduce_max_sync(0xffffffffu, guard_below);
    float f = a.c;
    if constexpr (BITS == 8) f = logit_factor(a.c * group_scale(a.kv.k_scale, s, (key0 + key_group * 32) & ~(kScaleTokens - 1), (pool_at + key_group * 32) & ~(kScaleTokens - 1), pool_rows), 1.f);
    const uint64_t ff = pack2(f, f);
    float sum[2][2] = {}, lost[2][2] = {};
#pragma unroll 1
    for (int stage = 0; stage < stages; ++stage) {
      const int slot = stage % kStages;
      if (in_group < kGroupRows) sm.below[row_group][slot][in_group] = -lse2[0];
      lse2[0] = lse2[1];
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      asm volatile("bar.sync %0, %1;" ::"r"(1 + row_group), "n"(kGroupThreads) : "memory");   // the stage is there, and the one before it is read
      if (stage + 2 < stages) lse2[1] = fetch((stage + 2) % kStages);
      asm volatile("cp.async.commit_group;" ::: "memory");
      uint64_t part[2][2] = {};                           // pairs: of either of the thread's rows of eight
      // Products of some eights of rows, one instruction at a time (kProducts): they are issued in turns with the exponentials of the rows
      // before, so that neither unit waits while all warps want the other.
      constexpr int kStep = T::STEP, kSteps = kGroupRows / 8 / kStep, kChains = 2 * kStep, kProducts = 2 * T::BLOCKS * kChains;
      float z[2][kStep][2][4];
      uint4 q[kStep];
      auto product = [&](int step, int i) {
        const int b = i / (2 * kChains), second = i / kChains & 1, j = i % kChains >> 1, kt = i & 1;
        float (&to)[4] = z[step & 1][j][kt];
        if (kt == 0 && second == 0)
          q[j] = *reinterpret_cast<const uint4*>(group_rows + slot * T::QSTAGE + row_chunk<T>((step * kStep + j) * 8 + (lane >> 2), 4 * b + c));
        if (i < kChains) mma_first(to, k[kt][b][0][0], k[kt][b][1][0], k[kt][b][0][1], k[kt][b][1][1], q[j].x, q[j].y);
        else if (second == 0) mma(to, k[kt][b][0][0], k[kt][b][1][0], k[kt][b][0][1], k[kt][b][1][1], q[j].x, q[j].y);
        else mma(to, k[kt][b][0][2], k[kt][b][1][2], k[kt][b][0][3], k[kt][b][1][3], q[j].z, q[j].w);
      };
#pragma unroll
      for (int i = 0; i < kProducts; ++i) product(0, i);
#pragma unroll
      for (int step = 0; step < kSteps; ++step) {
        const int rr = group_first + stage * kRows + step * 8 * kStep;
        float x[kStep][2][4];
#pragma unroll
        for (int j = 0; j < kStep; ++j) {
          const uint64_t below = *reinterpret_cast<const uint64_t*>(&sm.below[row_group][slot][(step * kStep + j) * 8 + 2 * c]);
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              unpack2(fma2(pack2(z[step & 1][j][kt][2 * h], z[step & 1][j][kt][2 * h + 1]), ff, below), x[j][kt][2 * h], x[j][kt][2 * h + 1]);
        }
#pragma unroll
        for (int i = 0; i < 8 * kStep; ++i) {
          if (step + 1 < kSteps) {
#pragma unroll
            for (int n = 0; n < kProducts / (8 * kStep); ++n) product(step + 1, i * (kProducts / (8 * kStep)) + n);
          }
          float& e = x[i >> 3][i >> 2 & 1][i & 3];
          asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+f"(e));
        }
        if (rr < guard_below) {
#pragma unroll
          for (int j = 0; j < kStep; ++j)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (rr + 8 * j + 2 * c + (e & 1) < from[kt][e >> 1]) x[j][kt][e] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < kStep; ++j)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int h = 0; h < 2; ++h) part[kt][h] = add2(part[kt][h], pack2(x[j][kt][2 * h], x[j][kt][2 * h + 1]));
      }
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float u, v;
          unpack2(part[kt][h], u, v);
          const float y = __fsub_rn(u + v, lost[kt][h]), t = __fadd_rn(sum[kt][h], y);
          lost[kt][h] = __fsub_rn(__fsub_rn(t, sum[kt][h]), y);
          sum[kt][h] = t;
        }
    }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x = sum[kt][h];
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        if (c == 0) sm.sums[row_group][key_group * 32 + kt * 16 + h * 8 + (lane >> 2)] = x;
      }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    if (books) {
      float got = 0.f;
#pragma unroll
      for (int g = 0; g < kRowGroups; ++g) got += sm.sums[g][threadIdx.x];
      book(w, (int64_t)pool_at + threadIdx.x, held, got, own, span.fresh, span.fresh_row);
    }
    __syncthreads();                                      // before the next item's rows and sums
    cur.at += stages + 1;
    ++cur.tile;
  }
}

template <int D, int BITS>
int32_t launch(const WeighArgs& w, int sm_count, cudaStream_t stream) {
  constexpr int kBytes = kRowGroups * kStages * Traits<D, BITS>::QSTAGE;
  static ContextSet done;
  const int32_t st = allow_shared_memory(reinterpret_cast<const void*>(weigh_prompt_kernel<D, BITS>), kBytes, done);
  if (st != SPF_OK) return st;
  weigh_prompt_kernel<D, BITS><<<sm_count, kThreads, kBytes, stream>>>(w);
  SPF_CUDA_CHECK(cudaGetLastError());
  return SPF_OK;
}

}  // namespace

int32_t weigh_prompt_launch(const WeighArgs& w, int head_dim, int sm_count, cudaStream_t stream) {
  const bool d64 = head_dim == 64;
  switch (w.a.kv.bits) {
    case 4: return d64 ? launch<64, 4>(w, sm_count, stream) : launch<128, 4>(w, sm_count, stream);
    case 8: return d64 ? launch<64, 8>(w, sm_count, stream) : launch<128, 8>(w, sm_count, stream);
    default: return d64 ? launch<64, 16>(w, sm_count, stream) : launch<128, 16>(w, sm_count, stream);
  }
}

}  // namespace spf
