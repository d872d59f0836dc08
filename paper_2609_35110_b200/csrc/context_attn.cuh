// Attention of query rows over keys and values that live elsewhere than the queries: in the pages of a cache, or in the states of an
// encoder.  Shared by the kernel for few rows (here) and the tensor-core kernel for many (context_attn_sm100.cuh).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>

#include "cache_kernels.cuh"
#include "device_types.cuh"
#include "ptx_sm100.cuh"

namespace sol {

// Keys and values: pages of a cache, or rows of packed contexts.
struct KeysDev {
  PagedDev c;                   // paged; contexts use k, v, ks, vs (strides {-, token, head}) and kv_heads only
  const int* begins;            // contexts: first row and length per sequence
  const int* lens;
  long long total_rows;         // contexts: rows of k and v
  const int* streams;           // paged: entry e of the batch is stream streams[e], or stream e if nullptr
  const uint8_t* mask;          // paged: row `stream` at mask_stride; contexts: one byte per row; nullptr: all valid
  long long mask_stride;
};

// Queries: sequences of a plan (schedule order), or one row per entry of a batch.
struct QueriesDev {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  long long q_tok, q_head, o_tok, o_head;
  const SeqDev* seqs;           // nullptr: entry e is row e
  const int* cum_tok;           // tokens of the sequences before each one in the schedule
  int n_seqs;                   // sequences, or entries
  int group;                    // query heads per K/V head; rows of a K/V head are (token, head in group), head fastest
  int causal;                   // 0, or tokens per block: row i sees the keys below N - n + (i / causal + 1) * causal
  float scale_log2;
};

// What one entry attends to.
struct Span {
  const uint8_t* mask;          // of key 0, or nullptr
  const int* table;             // paged
  long long begin;              // contexts: first row
  int n;                        // keys (paged: the tokens of the stream)
  int cap;                      // keys at or beyond this one do not count (what the mask row says nothing of)
  bool idle;                    // the entry names no stream: its rows stay as they are
};

template <bool kPaged>
__device__ __forceinline__ Span find_span(const KeysDev& d, int entry) {
  Span s{};
  if (kPaged) {
    const long long stream = d.streams != nullptr ? d.streams[entry] : entry;
    s.idle = stream < 0 || stream >= d.c.n_streams;
    if (s.idle) return s;
    s.n = (int)stream_tokens(d.c, stream);
    s.table = d.c.table + stream * d.c.width;
    s.mask = d.mask != nullptr ? d.mask + stream * d.mask_stride : nullptr;
    s.cap = s.mask != nullptr && d.mask_stride < s.n ? (int)d.mask_stride : s.n;
  } else {
    const long long b = d.begins[entry], n = d.lens[entry];
    s.begin = b < 0 ? 0 : b < d.total_rows ? b : d.total_rows;
    const long long left = d.total_rows - s.begin;
    s.n = (int)(n < 0 ? 0 : n < left ? n : left);
    s.cap = s.n;
    s.mask = d.mask != nullptr ? d.mask + s.begin : nullptr;
  }
  return s;
}

// Keys below this one count for token i of n new ones.
__device__ __forceinline__ int key_limit(const Span& s, int n_new, int i, int causal) {
  if (causal == 0) return s.cap;
  const long long lim = (long long)s.n - n_new + ((long long)(i / causal) + 1) * causal;
  return lim < 0 ? 0 : lim < s.cap ? (int)lim : s.cap;
}

// Units of `rows` (token, head) rows: sequence s of the schedule starts at unit cum_tok[s] * group / rows + s.  That leaves every
// sequence room for its ceil(n * group / rows) units without a running sum, and is found by bisection; up to one unit per
// sequence stays empty.
__device__ __forceinline__ int find_sequence(const QueriesDev& a, long long unit, int rows, long long* first) {
  int lo = 0, hi = a.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((long long)a.cum_tok[mid] * a.group / rows + mid <= unit) lo = mid; else hi = mid - 1;
  }
  *first = (long long)a.cum_tok[lo] * a.group / rows + lo;
  return lo;
}

// ---------------------------------------------------------------------------------------------
// Few query rows per K/V head (one token per stream, its heads that share the K/V head; a small chunk).  Bound by reading K and V
// once, of which latency leaves a fifth: 24 streams of 77 to 12,736 tokens, 40 / 8 heads x 128, masked, 0.567 GB: 108 us with the join in
// ten calls after a pause, 114 to 120 in a run (4.9 TB/s; 88 at the copy bandwidth); 12 warps per SM with two blocks of 16 keys in flight
// use 40 % of the issue slots (530 instructions per block), and wait for K and V as long as for their own instructions.  24 rows x 40 heads x 128 against 77 to 491 states,
// 0.140 GB: 31 us.
// A unit is up to 16 rows, the height of an mma.sync tile (m16n8k16); a CTA of four warps takes a unit and a range of
// keys, a warp 16 keys at a time.  The tensor core is there for the grouped heads: on the FMA pipes 16 rows would cost 16 x
// 256 operations per key and bind long before HBM does; a tcgen05 tile has 128 rows, of which 16 or fewer would be filled, and
// its operands would have to go through shared memory.
//
// Every warp has a ring of its own in shared memory that cp.async fills, some blocks ahead (rows padded by 16 bytes, so that the eight
// rows of an ldmatrix lie in different banks); no barrier but the warp's.  Masked keys are not read: their place is zeros, whatever
// the cache holds there.  K goes to the tensor core as it lies, V through the transposing ldmatrix.
//
// Three CTAs of four warps per SM, two blocks in flight per warp (D = 128).  With direct loads into operand registers the 24 streams took
// 177 us, with three blocks and two CTAs 164.
//
// Softmax in fp32 against a reference per row that moves only when a score exceeds it by more than 2^8.  P is held as two bf16 parts,
// most of p and what that leaves, whose products with V are added: the tensor core has time (48 of its instructions per 16
// keys; HBM allows 350 cycles for them), and the error is then the output's own rounding (0.0017 relative, 0.0020 with one
// part).  Keys are split over CTAs when there are few units; the parts are
// joined in a fixed order.
// ---------------------------------------------------------------------------------------------
constexpr int kFewRows = 16, kFewWarps = 4, kFewThreads = 32 * kFewWarps, kFewResident = 3;

template <int D>
struct FewSmem {
  static constexpr int kPitch = D * 2 + 16;               // bytes of a row
  static constexpr int kBlock = 16 * kPitch;              // 16 keys of K, or of V
  static constexpr int kStages = D == 128 ? 2 : 4;
  static constexpr int kRing = kStages * 2 * kBlock;      // per warp
  static constexpr int kOffValid = kFewWarps * kRing;     // validity of the keys of a stage, 32 bits per warp and stage
  static constexpr int kOffStats = kOffValid + kFewWarps * kStages * 4;
  static constexpr int kBytes = (kOffStats + kFewWarps * kFewRows * 12 + 15) / 16 * 16;
  static_assert(kRing >= kFewRows * (D + 4) * 4, "a warp's partial rows replace its ring at the end");
};

struct FewArgs {
  QueriesDev a;
  KeysDev d;
  int n_split;
  long long units;              // per K/V head
  float* partial;               // [kv_head][unit][split][16][D + 4], or nullptr: one split
};

// Which rows unit `unit` of a K/V head holds: entry of the batch, new tokens of it, first (token, head) row, its first token.
struct FewUnit {
  int entry, n_tok, row0;
  long long tok0;
};
__device__ __forceinline__ FewUnit find_few_rows(const QueriesDev& a, long long unit) {
  if (a.seqs != nullptr) {
    long long first;
    const SeqDev& sq = a.seqs[find_sequence(a, unit, kFewRows, &first)];
    return {sq.seq_id, sq.n_tokens, (int)(unit - first) * kFewRows, sq.tok_start};
  }
  const int per = (a.group + kFewRows - 1) / kFewRows, entry = (int)(unit / per);
  return {entry, 1, (int)(unit % per) * kFewRows, entry};
}

__device__ __forceinline__ void mma_bf16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int D, bool kPaged>
__global__ void __launch_bounds__(kFewThreads, kFewResident) few_rows_kernel(const __grid_constant__ FewArgs p) {
  using L = FewSmem<D>;
  extern __shared__ __align__(16) uint8_t few_smem[];
  chained_wait();
  chained_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;

  // ---- which rows, which keys
  const int split = blockIdx.x % p.n_split;
  const long long rest = blockIdx.x / p.n_split;
  const int kv_head = (int)(rest % p.d.c.kv_heads);
  const long long unit = rest / p.d.c.kv_heads;
  const auto [entry, n_tok, row0, tok0] = find_few_rows(p.a, unit);
  const int n_rows = min(kFewRows, n_tok * p.a.group - row0);
  if (n_rows <= 0) return;
  const Span sp = find_span<kPaged>(p.d, entry);
  if (sp.idle) return;

  // ---- the two rows of this lane's quad: tile rows g and g + 8
  int limit[2];
  uint32_t q[D / 16][4];                                // operand registers: [dims 16 k + 2 c, + 1, then + 8][row]
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int row = row0 + g + 8 * r;
    const bool there = g + 8 * r < n_rows;
    const int tok = there ? row / p.a.group : 0, h = there ? row % p.a.group : 0;
    limit[r] = there ? key_limit(sp, n_tok, tok, p.a.causal) : 0;
    const __nv_bfloat16* src = p.a.q + (tok0 + tok) * p.a.q_tok + ((long long)kv_head * p.a.group + h) * p.a.q_head + 2 * c;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int half = 0; half < 2; ++half)
        q[k][2 * half + r] = there ? *reinterpret_cast<const unsigned int*>(src + 16 * k + 8 * half) : 0u;
  }
  const int last_tok = (row0 + n_rows - 1) / p.a.group;
  const int most = key_limit(sp, n_tok, last_tok, p.a.causal);            // limits grow with the token
  const int least = key_limit(sp, n_tok, row0 / p.a.group, p.a.causal);
  // this CTA's blocks of 16 keys: whole turns of its four warps
  const int blocks = (most + 15) >> 4;
  const int per_split = ((blocks + p.n_split - 1) / p.n_split + kFewWarps - 1) / kFewWarps * kFewWarps;
  const int b_end = (int)min((long long)blocks, (long long)(split + 1) * per_split);

  // ---- the warp's ring
  const uint32_t ring = smem_u32(few_smem) + warp * L::kRing;
  uint32_t* valid_of = reinterpret_cast<uint32_t*>(few_smem + L::kOffValid) + warp * L::kStages;
  const int b_first = split * per_split + warp;
  constexpr int kChunks16 = D / 8;                      // 16-byte chunks of a row
  const int chunk = lane % kChunks16, row_first = lane / kChunks16;
  constexpr int kRowStep = 32 / kChunks16;
  const __nv_bfloat16* kh = p.d.c.k + kv_head * p.d.c.ks[2] + chunk * 8;
  const __nv_bfloat16* vh = p.d.c.v + kv_head * p.d.c.vs[2] + chunk * 8;
  const long long k_step = kRowStep * p.d.c.ks[1], v_step = kRowStep * p.d.c.vs[1];
  // What a block needs before its loads can start is fetched a turn earlier, ahead of V of the turn's block (behind it: 24 streams 122 us
  // instead of 116): its page, and the mask's word on its keys.  Its place among the pages moves with it (four blocks a turn), without a
  // division.
  const int page = kPaged ? p.d.c.page : 1, page_cols = 16 * kFewWarps / page, page_rows = 16 * kFewWarps % page;
  int col = kPaged ? b_first * 16 / page : 0, in_page = kPaged ? b_first * 16 % page : 0;
  int page_ahead = 0, row_ahead = 0;
  bool on_ahead = false;
  auto look_up = [&](int b) {
    if (b >= b_end) return;
    if (kPaged) {
      page_ahead = sp.table[col];
      row_ahead = in_page;
      col += page_cols;
      in_page += page_rows;
      if (in_page >= page) { in_page -= page; ++col; }
    }
    const int key = b * 16 + (lane & 15);
    on_ahead = key < most && (sp.mask == nullptr || sp.mask[key] != 0);
  };
  // K of block b into a stage, then V of the same block: two steps, because K's place is free as soon as the scores are computed
  uint32_t v_valid = 0;
  const __nv_bfloat16* v_next = nullptr;
  auto copy_rows = [&](uint32_t dst, const __nv_bfloat16* src, long long step, uint32_t valid, const __nv_bfloat16* safe) {
    if (valid == 0xffffu) {
#pragma unroll
      for (int i = 0; i < 16 / kRowStep; ++i, src += step) cp_async_16(dst + i * kRowStep * L::kPitch, src, 16);
    } else {
      valid >>= row_first;
#pragma unroll
      for (int i = 0; i < 16 / kRowStep; ++i, src += step) {
        const bool on = (valid >> (i * kRowStep)) & 1u;
        // (a key that is not read keeps its address inside a page; behind the last row of a context there may be no memory)
        cp_async_16(dst + i * kRowStep * L::kPitch, kPaged || on ? src : safe, on ? 16 : 0);
      }
    }
  };
  auto fetch_k = [&](int b, int stage) {
    if (b < b_end) {
      uint32_t valid = __ballot_sync(0xffffffffu, on_ahead) & 0xffffu;
      if (lane == 0) valid_of[stage] = valid;
      long long krow, vrow;
      if (kPaged) {                                     // (a page holds whole blocks: its size is a multiple of 16)
        const bool there = page_ahead >= 0 && page_ahead < p.d.c.n_pages;
        const long long at = there ? page_ahead : 0;    // no such page: zeros, and an address that there is
        krow = at * p.d.c.ks[0] + row_ahead * p.d.c.ks[1];
        vrow = at * p.d.c.vs[0] + row_ahead * p.d.c.vs[1];
        if (!there) valid = 0;
      } else {
        krow = (sp.begin + b * 16) * p.d.c.ks[1];
        vrow = (sp.begin + b * 16) * p.d.c.vs[1];
      }
      v_valid = valid;
      v_next = vh + vrow + row_first * p.d.c.vs[1];
      copy_rows(ring + stage * 2 * L::kBlock + row_first * L::kPitch + chunk * 16, kh + krow + row_first * p.d.c.ks[1], k_step, valid, p.d.c.k);
    }
    cp_async_commit();
  };
  auto fetch_v = [&](int b, int stage) {
    if (b < b_end) {
      look_up(b + kFewWarps);
      copy_rows(ring + stage * 2 * L::kBlock + L::kBlock + row_first * L::kPitch + chunk * 16, v_next, v_step, v_valid, p.d.c.v);
    }
    cp_async_commit();
  };
  look_up(b_first);
#pragma unroll
  for (int s = 0; s < L::kStages; ++s) {
    fetch_k(b_first + s * kFewWarps, s);
    fetch_v(b_first + s * kFewWarps, s);
  }

  float o[D / 8][4];
#pragma unroll
  for (int t = 0; t < D / 8; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[t][e] = 0.f;
  float m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};
  bool seen[2] = {false, false};
  const float sc = p.a.scale_log2;
  // an ldmatrix lane's row: of K, keys (lane & 7) + 8 (lane >> 4), dims + 8 for odd (lane >> 3); of V, keys lane & 15, dims + 8 (lane >> 4)
  const uint32_t k_lane = ((lane & 7) + 8 * (lane >> 4)) * L::kPitch + ((lane >> 3) & 1) * 16;
  const uint32_t v_lane = (lane & 15) * L::kPitch + (lane >> 4) * 16;

  int stage = 0;
#pragma unroll 1
  for (int b = b_first; b < b_end; b += kFewWarps) {
    cp_async_wait<2 * L::kStages - 1>();                // K of this block is there
    __syncwarp();
    const int key0 = b * 16;
    const uint32_t k_at = ring + stage * 2 * L::kBlock + k_lane, v_at = ring + stage * 2 * L::kBlock + L::kBlock + v_lane;
    const uint32_t valid = valid_of[stage];
    // ---- scores: [t] keys 8 t + 2 c, + 1; entries 0, 1 of row g, 2, 3 of row g + 8 (two chains of products each)
    float s[2][4], s2[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] = s2[t][e] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; k += 2) {
      uint32_t x[4], y[4];
      ldmatrix_x4(k_at + k * 32, x);
      ldmatrix_x4(k_at + k * 32 + 32, y);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        mma_bf16_16816(s[t], q[k][0], q[k][1], q[k][2], q[k][3], x[2 * t], x[2 * t + 1]);
        mma_bf16_16816(s2[t], q[k + 1][0], q[k + 1][1], q[k + 1][2], q[k + 1][3], y[2 * t], y[2 * t + 1]);
      }
    }
    __syncwarp();
    fetch_k(b + L::kStages * kFewWarps, stage);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] += s2[t][e];
    if (key0 + 16 > least && least < most) {            // the rows do not see the same keys
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = 8 * t + 2 * c + (e & 1);
          const bool on = ((valid >> key) & 1u) != 0 && key0 + key < limit[e >> 1];
          if (!on) s[t][e] = -CUDART_INF_F;
          seen[e >> 1] = seen[e >> 1] || on;
        }
    } else {
      if (valid != 0xffffu) {
        const uint32_t mine = valid >> (2 * c);         // bits 0, 1, 8, 9: this lane's keys
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (((mine >> (8 * t + e)) & 1u) == 0) s[t][e] = s[t][2 + e] = -CUDART_INF_F;
      }
      seen[0] = seen[1] = seen[0] || valid != 0;        // (rows that the unit does not have: not written)
    }
    // ---- the rows' references: the largest score of the first block with a valid key, moved when one exceeds it by more than 2^8
    float x[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      x[r] = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
      x[r] = fmaxf(x[r], __shfl_xor_sync(0xffffffffu, x[r], 1));
      x[r] = fmaxf(x[r], __shfl_xor_sync(0xffffffffu, x[r], 2));
    }
    const bool move0 = (x[0] - m[0]) * sc > 8.f, move1 = (x[1] - m[1]) * sc > 8.f;
    if (__any_sync(0xffffffffu, move0 || move1)) {
      const float f0 = move0 ? ex2_approx((m[0] - x[0]) * sc) : 1.f, f1 = move1 ? ex2_approx((m[1] - x[1]) * sc) : 1.f;
      if (move0) m[0] = x[0];
      if (move1) m[1] = x[1];
#pragma unroll
      for (int t = 0; t < D / 8; ++t) {
        o[t][0] *= f0; o[t][1] *= f0;
        o[t][2] *= f1; o[t][3] *= f1;
      }
      l[0] *= f0;
      l[1] *= f1;
    }
    const float base[2] = {m[0] == -CUDART_INF_F ? 0.f : m[0] * sc, m[1] == -CUDART_INF_F ? 0.f : m[1] * sc};   // (nothing valid yet: 2^-inf)
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float p0 = ex2_approx(fmaf(s[t][2 * r], sc, -base[r])), p1 = ex2_approx(fmaf(s[t][2 * r + 1], sc, -base[r]));
        l[r] += p0 + p1;
        // (the larger part stays below p, so that both are positive: an infinite value times them is not inf - inf, nor inf * 0)
        const uint32_t h0 = __float_as_uint(p0 * 0.99609375f) & 0xffff0000u, h1 = __float_as_uint(p1 * 0.99609375f) & 0xffff0000u;
        hi[2 * t + r] = __byte_perm(h0, h1, 0x7632);
        lo[2 * t + r] = pack_bf16x2(p0 - __uint_as_float(h0), p1 - __uint_as_float(h1));
      }
    // ---- O += P V
    cp_async_wait<2 * L::kStages - 1>();                // V of this block is there
    __syncwarp();
#pragma unroll
    for (int j = 0; j < D / 8; j += 2) {
      uint32_t x[4];
      ldmatrix_x4_trans(v_at + j * 16, x);
      mma_bf16_16816(o[j], hi[0], hi[1], hi[2], hi[3], x[0], x[1]);
      mma_bf16_16816(o[j + 1], hi[0], hi[1], hi[2], hi[3], x[2], x[3]);
      mma_bf16_16816(o[j], lo[0], lo[1], lo[2], lo[3], x[0], x[1]);
      mma_bf16_16816(o[j + 1], lo[0], lo[1], lo[2], lo[3], x[2], x[3]);
    }
    __syncwarp();
    fetch_v(b + L::kStages * kFewWarps, stage);
    if (++stage == L::kStages) stage = 0;
  }
  cp_async_wait<0>();
  __syncwarp();

  // ---- the four warps' parts: rows in place of the warp's ring, statistics beside them
  auto rows_of = [&](int w) { return reinterpret_cast<float*>(few_smem + w * L::kRing); };
  float* s_m = reinterpret_cast<float*>(few_smem + L::kOffStats);
  float* s_l = s_m + kFewWarps * kFewRows;
  int* s_seen = reinterpret_cast<int*>(s_l + kFewWarps * kFewRows);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    int any = seen[r];
    any |= __shfl_xor_sync(0xffffffffu, any, 1);
    any |= __shfl_xor_sync(0xffffffffu, any, 2);
    const int row = g + 8 * r;
    if (c == 0) {
      s_m[warp * kFewRows + row] = m[r];
      s_l[warp * kFewRows + row] = l[r];
      s_seen[warp * kFewRows + row] = any;
    }
    if (row < n_rows)
#pragma unroll
      for (int j = 0; j < D / 8; ++j)
        *reinterpret_cast<float2*>(rows_of(warp) + row * (D + 4) + 8 * j + 2 * c) = make_float2(o[j][2 * r], o[j][2 * r + 1]);
  }
  __syncthreads();
  constexpr int kChunks = D / 8;                                            // a thread takes 8 dims of a row
  for (int x = threadIdx.x; x < n_rows * kChunks; x += kFewThreads) {
    const int row = x / kChunks, d0 = (x % kChunks) * 8;
    float top = -CUDART_INF_F;
    int any = 0;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      top = fmaxf(top, s_m[w * kFewRows + row]);
      any |= s_seen[w * kFewRows + row];
    }
    float sum = 0.f, acc[8] = {};
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      if (!s_seen[w * kFewRows + row]) continue;
      const float mw = s_m[w * kFewRows + row], f = mw == top ? 1.f : ex2_approx((mw - top) * sc);
      sum = fmaf(s_l[w * kFewRows + row], f, sum);
      const float* src = rows_of(w) + row * (D + 4) + d0;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = fmaf(src[e], f, acc[e]);
    }
    if (p.partial != nullptr) {
      float* dst = p.partial + (((kv_head * p.units + unit) * p.n_split + split) * kFewRows + row) * (D + 4);
      *reinterpret_cast<float4*>(dst + d0) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      *reinterpret_cast<float4*>(dst + d0 + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
      if (d0 == 0) *reinterpret_cast<float4*>(dst + D) = make_float4(top, sum, any ? 1.f : 0.f, 0.f);
    } else {
      const float inv = any ? 1.f / sum : 0.f;                              // no valid key: zeros
      const int r = row0 + row;
      __nv_bfloat16* dst = p.a.out + (tok0 + r / p.a.group) * p.a.o_tok + ((long long)kv_head * p.a.group + r % p.a.group) * p.a.o_head + d0;
      uint4 y = make_uint4(0, 0, 0, 0);
      if (any) y = make_uint4(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv),
                              pack_bf16x2(acc[4] * inv, acc[5] * inv), pack_bf16x2(acc[6] * inv, acc[7] * inv));
      *reinterpret_cast<uint4*>(dst) = y;
    }
  }
}

// Joins the parts of split keys.  Rows of partial results: D values, maximum, sum, "has a valid key".  A warp's lanes look at the
// statistics of 32 parts at once; then a lane sums 8 dims over every second (D = 128) or fourth part, with weights that come by
// shuffle, so that the loads of the values do not wait for one another.  All sums are in a fixed order.
__device__ __forceinline__ float largest_part(const float* stats, long long step, int n_parts, bool* any) {
  float top = -CUDART_INF_F;
  bool some = false;
  for (int s = threadIdx.x & 31; s < n_parts; s += 32) {
    const float4 t = *reinterpret_cast<const float4*>(stats + s * step);
    top = fmaxf(top, t.x);
    some = some || t.z != 0.f;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  *any = __any_sync(0xffffffffu, some);
  return top;
}

// Parts [begin, end) of a row, weighted against `top`; every lane ends with the sum of weights and the 8 dims at (lane % (D / 8)) * 8.
template <int D>
__device__ __forceinline__ void sum_parts(const float* mine, long long step, int begin, int end, float top, float scale_log2, float& sum, float (&acc)[8]) {
  constexpr int kChunks = D / 8, kTeams = 32 / kChunks;
  const int lane = threadIdx.x & 31, d0 = lane % kChunks * 8, team = lane / kChunks;
  sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  for (int s0 = begin; s0 < end; s0 += 32) {
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (s0 + lane < end) t = *reinterpret_cast<const float4*>(mine + (s0 + lane) * step + D);
    const float weight = t.z == 0.f ? 0.f : t.x == top ? 1.f : ex2_approx((t.x - top) * scale_log2);
    if (t.z != 0.f) sum = fmaf(t.y, weight, sum);
    const unsigned there = __ballot_sync(0xffffffffu, t.z != 0.f);         // (what a part without a valid key holds is not looked at)
#pragma unroll 4
    for (int j = 0; j < 32; j += kTeams) {
      if (s0 + j >= end) break;
      const float f = __shfl_sync(0xffffffffu, weight, j + team);
      if ((there >> (j + team)) & 1u) {
        const float* v = mine + (s0 + j + team) * step + d0;
        const float4 a = *reinterpret_cast<const float4*>(v), b = *reinterpret_cast<const float4*>(v + 4);
        acc[0] = fmaf(a.x, f, acc[0]); acc[1] = fmaf(a.y, f, acc[1]); acc[2] = fmaf(a.z, f, acc[2]); acc[3] = fmaf(a.w, f, acc[3]);
        acc[4] = fmaf(b.x, f, acc[4]); acc[5] = fmaf(b.y, f, acc[5]); acc[6] = fmaf(b.z, f, acc[6]); acc[7] = fmaf(b.w, f, acc[7]);
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (o >= kChunks)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], o);
  }
}

// 8 dims of a joined row; zeros where there is no valid key.
__device__ __forceinline__ void store_joined(__nv_bfloat16* dst, const float (&acc)[8], float sum, bool any) {
  const float inv = 1.f / sum;
  uint4 y = make_uint4(0, 0, 0, 0);
  if (any) y = make_uint4(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv),
                          pack_bf16x2(acc[4] * inv, acc[5] * inv), pack_bf16x2(acc[6] * inv, acc[7] * inv));
  *reinterpret_cast<uint4*>(dst) = y;
}

constexpr int kJoinWarps = 8, kJoinFewWarps = 4;

// After few_rows_kernel.  Grid: units x K/V heads, rows of a unit.  With many parts a CTA takes a row, a quarter of the parts per warp:
// a long past has some hundred, and few rows (one stream of 111,856 keys, 15 rows x 8 K/V heads, attention and join: 167 us with
// all rows of a unit in one CTA, 112 us so).  With few parts a warp takes a row (kWarps = 1).  960 units of 12 rows,
// 4 parts: 500 us with a CTA per row, 484 with a warp; 192 of 5 rows, 13 parts: 111 and 115; so the line is drawn at 8.
template <int D, bool kPaged, int kWarps>
__global__ void __launch_bounds__(32 * kJoinFewWarps) join_few_kernel(const __grid_constant__ FewArgs p) {
  __shared__ float part_acc[kWarps][D], part_sum[kWarps];
  chained_wait();
  chained_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int kv_head = (int)(blockIdx.x / p.units), row = blockIdx.y * (kJoinFewWarps / kWarps) + (kWarps == 1 ? warp : 0);
  const long long unit = blockIdx.x % p.units;
  const auto [entry, n_tok, row0, tok0] = find_few_rows(p.a, unit);
  if (kPaged) {
    const long long stream = p.d.streams != nullptr ? p.d.streams[entry] : entry;
    if (stream < 0 || stream >= p.d.c.n_streams) return;
  }
  if (row >= n_tok * p.a.group - row0) return;
  const int d0 = lane % (D / 8) * 8;
  const long long step = (long long)kFewRows * (D + 4);
  const float* mine = p.partial + ((long long)blockIdx.x * p.n_split * kFewRows + row) * (D + 4);
  bool any;
  const float top = largest_part(mine + D, step, p.n_split, &any);
  const int each = (p.n_split + kWarps - 1) / kWarps, begin = kWarps == 1 ? 0 : min(warp * each, p.n_split);
  float sum, acc[8];
  sum_parts<D>(mine, step, begin, min(begin + each, p.n_split), top, p.a.scale_log2, sum, acc);
  if (kWarps > 1) {
    if (lane < D / 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) part_acc[warp][d0 + e] = acc[e];
      if (lane == 0) part_sum[warp] = sum;
    }
    __syncthreads();                                       // (the rows of a CTA are one: all its warps are here)
    if (warp > 0) return;
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      sum += part_sum[w];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += part_acc[w][d0 + e];
    }
  }
  if (lane >= D / 8) return;
  const int r = row0 + row;
  store_joined(p.a.out + (tok0 + r / p.a.group) * p.a.o_tok + ((long long)kv_head * p.a.group + r % p.a.group) * p.a.o_head + d0, acc, sum, any);
}

// After context_attn_kernel: the units whose keys it split are listed on the device.  A warp per row of one.
struct JoinUnit {
  long long tok0;
  int t0, n_tok;                // first new token of the unit; new tokens of the sequence (0: nothing to join)
  int kv_head;
  int first_part, n_parts;      // its partial rows
  int unused;
};
struct JoinArgs {
  QueriesDev a;
  int rows_per_unit;
  const float* partial;
  const JoinUnit* list;
  const int* count;
  const unsigned int* status;   // not zero: a wait ran out, now or earlier, and list and count may never have been written
};

template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps) join_units_kernel(const __grid_constant__ JoinArgs p) {
  chained_wait();
  chained_next();
  const int count = *p.count;
  if (count <= 0 || *p.status != 0) return;
  const long long all = (long long)count * p.rows_per_unit;
  for (long long x = (long long)blockIdx.x * kJoinWarps + (threadIdx.x >> 5); x < all; x += (long long)gridDim.x * kJoinWarps) {
    const JoinUnit u = p.list[x / p.rows_per_unit];
    const int row = (int)(x % p.rows_per_unit), tok = u.t0 + row / p.a.group;
    if (tok >= u.n_tok) continue;
    const long long step = (long long)p.rows_per_unit * (D + 4);
    const float* mine = p.partial + u.first_part * step + row * (D + 4);
    bool any;
    const float top = largest_part(mine + D, step, u.n_parts, &any);
    float sum, acc[8];
    sum_parts<D>(mine, step, 0, u.n_parts, top, p.a.scale_log2, sum, acc);
    const int lane = threadIdx.x & 31, d0 = lane * 8;
    if (lane < D / 8) store_joined(p.a.out + (u.tok0 + tok) * p.a.o_tok + ((long long)u.kv_head * p.a.group + row % p.a.group) * p.a.o_head + d0, acc, sum, any);
  }
}

}  // namespace sol
