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
// once.  A unit is up to 16 rows, the height of an mma.sync tile (m16n8k16); a CTA of four warps takes a unit and a range of
// keys, a warp 16 keys at a time.  The tensor core is there for the grouped heads: on the FMA pipes 16 rows would cost 16 x
// 256 operations per key and bind long before HBM does; a tcgen05 tile has 128 rows, of which 16 or fewer would be filled, and
// its operands would have to go through shared memory.
//
// Nothing is staged: lanes load 16 bytes of global memory straight into operand registers.  A product does not care for the order
// of the index that it sums over, so the K dims of a 32-dim step are assigned such that a lane's operand registers are eight
// neighbouring dims of one key: lane 4 g + c has dims 8 c .. 8 c + 7 of keys g and g + 8.  For P V the summed index is the key, two
// to a register: lane 4 g + c loads dims 8 g .. 8 g + 7 of keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9 and pairs them with byte permutes; output
// column g of product e is dim 8 g + e, which leaves a lane with 16 neighbouring dims of its two rows.
//
// Softmax in fp32 with a running maximum per row; P is rounded to bf16 for the product (its row sum is of the unrounded values), as
// in the dense kernel.  Keys are split over CTAs when there are few units; the parts are joined in a fixed order.
// ---------------------------------------------------------------------------------------------
constexpr int kFewRows = 16, kFewWarps = 4, kFewThreads = 32 * kFewWarps, kFewResident = 3;

struct FewArgs {
  QueriesDev a;
  KeysDev d;
  int n_split;
  long long units;              // per K/V head
  float* partial;               // [kv_head][unit][split][16][D + 4], or nullptr: one split
};

__device__ __forceinline__ void mma_bf16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <int D, bool kPaged>
__global__ void __launch_bounds__(kFewThreads, kFewResident) few_rows_kernel(const __grid_constant__ FewArgs p) {
  constexpr int kK = D / 32, kV = D / 64;               // 16-byte loads per key: of K by a quad, of V by eight lanes
  __shared__ float s_o[kFewWarps][kFewRows][D + 4];
  __shared__ float s_m[kFewWarps][kFewRows], s_l[kFewWarps][kFewRows];
  __shared__ int s_seen[kFewWarps][kFewRows];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;

  // ---- which rows, which keys
  const int split = blockIdx.x % p.n_split;
  const long long rest = blockIdx.x / p.n_split;
  const int kv_head = (int)(rest % p.d.c.kv_heads);
  const long long unit = rest / p.d.c.kv_heads;
  int entry, n_tok, row0;                               // of the batch; new tokens; first (token, head) row
  long long tok0;
  if (p.a.seqs != nullptr) {
    long long first;
    const SeqDev& sq = p.a.seqs[find_sequence(p.a, unit, kFewRows, &first)];
    entry = sq.seq_id;
    n_tok = sq.n_tokens;
    tok0 = sq.tok_start;
    row0 = (int)(unit - first) * kFewRows;
  } else {
    const int per = (p.a.group + kFewRows - 1) / kFewRows;
    entry = (int)(unit / per);
    n_tok = 1;
    tok0 = entry;
    row0 = (int)(unit % per) * kFewRows;
  }
  const int n_rows = min(kFewRows, n_tok * p.a.group - row0);
  if (n_rows <= 0) return;
  const Span sp = find_span<kPaged>(p.d, entry);
  if (sp.idle) return;

  // ---- the two rows of this lane's quad: tile rows g and g + 8
  int limit[2];
  uint4 q[2][kK];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int row = row0 + g + 8 * r;
    const bool there = g + 8 * r < n_rows;
    const int tok = there ? row / p.a.group : 0, h = there ? row % p.a.group : 0;
    limit[r] = there ? key_limit(sp, n_tok, tok, p.a.causal) : 0;
    const __nv_bfloat16* src = p.a.q + (tok0 + tok) * p.a.q_tok + ((long long)kv_head * p.a.group + h) * p.a.q_head + c * 8;
#pragma unroll
    for (int j = 0; j < kK; ++j) q[r][j] = there ? __ldg(reinterpret_cast<const uint4*>(src + j * 32)) : make_uint4(0, 0, 0, 0);
  }
  const int last_tok = (row0 + n_rows - 1) / p.a.group;
  const int most = key_limit(sp, n_tok, last_tok, p.a.causal);            // limits grow with the token
  const int least = key_limit(sp, n_tok, row0 / p.a.group, p.a.causal);
  // this CTA's blocks of 16 keys: whole turns of its four warps
  const int blocks = (most + 15) >> 4;
  const int per_split = ((blocks + p.n_split - 1) / p.n_split + kFewWarps - 1) / kFewWarps * kFewWarps;
  const int b_end = (int)min((long long)blocks, (long long)(split + 1) * per_split);

  float o[kV * 8][4];
#pragma unroll
  for (int t = 0; t < kV * 8; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[t][e] = 0.f;
  float m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};
  bool seen[2] = {false, false};
  const float sc = p.a.scale_log2;
  const __nv_bfloat16* kh = p.d.c.k + kv_head * p.d.c.ks[2] + c * 8;
  const __nv_bfloat16* vh = p.d.c.v + kv_head * p.d.c.vs[2] + g * 8;

  for (int b = split * per_split + warp; b < b_end; b += kFewWarps) {
    const int key0 = b * 16;
    // ---- where these 16 keys are (a page holds whole blocks: its size is a multiple of 16)
    long long krow, vrow;
    bool there = true;
    if (kPaged) {
      const int page = __ldg(sp.table + key0 / p.d.c.page), in_page = key0 % p.d.c.page;
      there = page >= 0 && page < p.d.c.n_pages;
      krow = page * p.d.c.ks[0] + in_page * p.d.c.ks[1];
      vrow = page * p.d.c.vs[0] + in_page * p.d.c.vs[1];
    } else {
      krow = (sp.begin + key0) * p.d.c.ks[1];
      vrow = (sp.begin + key0) * p.d.c.vs[1];
    }
    const bool whole = key0 + 16 <= most;
    uint4 kx[2][kK], vx[4][kV];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = g + 8 * t;
      const bool on = there && (whole || key0 + key < most);
      const __nv_bfloat16* src = kh + krow + key * p.d.c.ks[1];
#pragma unroll
      for (int j = 0; j < kK; ++j) kx[t][j] = on ? __ldg(reinterpret_cast<const uint4*>(src + j * 32)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int key = 2 * c + (t & 1) + 8 * (t >> 1);
      const bool on = there && (whole || key0 + key < most);
      const __nv_bfloat16* src = vh + vrow + key * p.d.c.vs[1];
#pragma unroll
      for (int j = 0; j < kV; ++j) vx[t][j] = on ? __ldg(reinterpret_cast<const uint4*>(src + j * 64)) : make_uint4(0, 0, 0, 0);
    }
    uint32_t valid = 0xffffu;
    if (sp.mask != nullptr) {
      const bool on = key0 + (lane & 15) < most && __ldg(sp.mask + key0 + (lane & 15)) != 0;
      valid = __ballot_sync(0xffffffffu, on) & 0xffffu;
      if (valid == 0) continue;
      // values of keys that do not count may be anything: they become zeros
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (((valid >> (2 * c + (t & 1) + 8 * (t >> 1))) & 1u) == 0)
#pragma unroll
          for (int j = 0; j < kV; ++j) vx[t][j] = make_uint4(0, 0, 0, 0);
    }
    // ---- scores: [t] keys 8 t + 2 c, + 1; entries 0, 1 of row g, 2, 3 of row g + 8
    float s[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] = 0.f;
#pragma unroll
      for (int j = 0; j < kK; ++j) {
        mma_bf16_16816(s[t], q[0][j].x, q[1][j].x, q[0][j].y, q[1][j].y, kx[t][j].x, kx[t][j].y);
        mma_bf16_16816(s[t], q[0][j].z, q[1][j].z, q[0][j].w, q[1][j].w, kx[t][j].z, kx[t][j].w);
      }
    }
    if (valid != 0xffffu || key0 + 16 > least) {
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
      seen[0] = seen[1] = true;
    }
    // ---- running maximum of the row, over the quad
    float scale[2];
    float base[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
      x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
      x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
      x = fmaxf(x, m[r]);
      base[r] = x == -CUDART_INF_F ? 0.f : x * sc;                          // (nothing valid yet: every term below is 2^-inf)
      scale[r] = x == m[r] ? 1.f : ex2_approx(m[r] * sc - base[r]);
      m[r] = x;
    }
    if (__any_sync(0xffffffffu, scale[0] != 1.f || scale[1] != 1.f)) {
#pragma unroll
      for (int t = 0; t < kV * 8; ++t) {
        o[t][0] *= scale[0]; o[t][1] *= scale[0];
        o[t][2] *= scale[1]; o[t][3] *= scale[1];
      }
      l[0] *= scale[0];
      l[1] *= scale[1];
    }
    uint32_t pa[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float p0 = ex2_approx(fmaf(s[t][2 * r], sc, -base[r])), p1 = ex2_approx(fmaf(s[t][2 * r + 1], sc, -base[r]));
        l[r] += p0 + p1;
        pa[2 * t + r] = pack_bf16x2(p0, p1);
      }
    // ---- O += P V
#pragma unroll
    for (int j = 0; j < kV; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t pick = (e & 1) ? 0x7632u : 0x5410u;
        const uint32_t b0 = __byte_perm(word(vx[0][j], e >> 1), word(vx[1][j], e >> 1), pick);
        const uint32_t b1 = __byte_perm(word(vx[2][j], e >> 1), word(vx[3][j], e >> 1), pick);
        mma_bf16_16816(o[j * 8 + e], pa[0], pa[1], pa[2], pa[3], b0, b1);
      }
  }

  // ---- the four warps' parts
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    int any = seen[r];
    any |= __shfl_xor_sync(0xffffffffu, any, 1);
    any |= __shfl_xor_sync(0xffffffffu, any, 2);
    const int row = g + 8 * r;
    if (c == 0) {
      s_m[warp][row] = m[r];
      s_l[warp][row] = l[r];
      s_seen[warp][row] = any;
    }
    if (row < n_rows)
#pragma unroll
      for (int j = 0; j < kV; ++j)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int e = 0; e < 8; e += 4)
            *reinterpret_cast<float4*>(&s_o[warp][row][j * 64 + (2 * c + half) * 8 + e]) =
                make_float4(o[j * 8 + e][2 * r + half], o[j * 8 + e + 1][2 * r + half], o[j * 8 + e + 2][2 * r + half], o[j * 8 + e + 3][2 * r + half]);
  }
  __syncthreads();
  constexpr int kChunks = D / 8;                                            // a thread takes 8 dims of a row
  for (int x = threadIdx.x; x < n_rows * kChunks; x += kFewThreads) {
    const int row = x / kChunks, d0 = (x % kChunks) * 8;
    float top = -CUDART_INF_F;
    int any = 0;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      top = fmaxf(top, s_m[w][row]);
      any |= s_seen[w][row];
    }
    float sum = 0.f, acc[8] = {};
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      if (!s_seen[w][row]) continue;
      const float f = s_m[w][row] == top ? 1.f : ex2_approx((s_m[w][row] - top) * sc);
      sum = fmaf(s_l[w][row], f, sum);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = fmaf(s_o[w][row][d0 + e], f, acc[e]);
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

// Joins the parts of split keys, in the order of the splits.  Rows of partial results: D values, maximum, sum, "has a valid key".
// One thread per 8 dims of a row; CTAs (unit and K/V head, 256 such pieces).  Whose rows a unit holds follows from its number (few rows), or was
// written down by who made them (kListed).
struct JoinUnit {
  long long tok0;
  int t0, n_tok;                // first new token of the unit; new tokens of the sequence (0: nothing to join)
  int kv_head;
  int unused;
};
struct JoinArgs {
  QueriesDev a;
  KeysDev d;
  int n_split, rows_per_unit;
  long long units;
  const float* partial;
  const JoinUnit* list;
};

template <int D, bool kPaged, bool kListed>
__global__ void __launch_bounds__(256) join_rows_kernel(const __grid_constant__ JoinArgs p) {
  int kv_head, n_tok;
  long long tok0, row0;
  if (kListed) {
    const JoinUnit u = p.list[blockIdx.x];
    kv_head = u.kv_head;
    n_tok = u.n_tok;
    tok0 = u.tok0;
    row0 = (long long)u.t0 * p.a.group;
  } else {
    int entry;
    kv_head = (int)(blockIdx.x / p.units);
    const long long unit = blockIdx.x % p.units;
    if (p.a.seqs != nullptr) {
      long long first;
      const SeqDev& sq = p.a.seqs[find_sequence(p.a, unit, p.rows_per_unit, &first)];
      entry = sq.seq_id;
      n_tok = sq.n_tokens;
      tok0 = sq.tok_start;
      row0 = (unit - first) * p.rows_per_unit;
    } else {
      const int per = (p.a.group + p.rows_per_unit - 1) / p.rows_per_unit;
      entry = (int)(unit / per);
      n_tok = 1;
      tok0 = entry;
      row0 = (unit % per) * p.rows_per_unit;
    }
    if (kPaged) {
      const long long stream = p.d.streams != nullptr ? p.d.streams[entry] : entry;
      if (stream < 0 || stream >= p.d.c.n_streams) return;
    }
  }
  const long long n_rows = min((long long)p.rows_per_unit, (long long)n_tok * p.a.group - row0);
  if (n_rows <= 0) return;
  constexpr int kChunks = D / 8;
  const float* part = p.partial + (long long)blockIdx.x * p.n_split * p.rows_per_unit * (D + 4);
  const int x = blockIdx.y * 256 + threadIdx.x;
  if (x < n_rows * kChunks) {
    const int row = x / kChunks, d0 = (x % kChunks) * 8;
    const float* mine = part + (long long)row * (D + 4);
    const long long step = (long long)p.rows_per_unit * (D + 4);
    float top = -CUDART_INF_F;
    bool any = false;
    for (int s = 0; s < p.n_split; ++s) {
      const float4 t = __ldg(reinterpret_cast<const float4*>(mine + s * step + D));
      top = fmaxf(top, t.x);
      any = any || t.z != 0.f;
    }
    float sum = 0.f, acc[8] = {};
#pragma unroll 4
    for (int s = 0; s < p.n_split; ++s) {
      const float4 t = __ldg(reinterpret_cast<const float4*>(mine + s * step + D));
      const float4 u = __ldg(reinterpret_cast<const float4*>(mine + s * step + d0)), v = __ldg(reinterpret_cast<const float4*>(mine + s * step + d0 + 4));
      if (t.z == 0.f) continue;
      const float f = t.x == top ? 1.f : ex2_approx((t.x - top) * p.a.scale_log2);
      sum = fmaf(t.y, f, sum);
      acc[0] = fmaf(u.x, f, acc[0]); acc[1] = fmaf(u.y, f, acc[1]); acc[2] = fmaf(u.z, f, acc[2]); acc[3] = fmaf(u.w, f, acc[3]);
      acc[4] = fmaf(v.x, f, acc[4]); acc[5] = fmaf(v.y, f, acc[5]); acc[6] = fmaf(v.z, f, acc[6]); acc[7] = fmaf(v.w, f, acc[7]);
    }
    const float inv = 1.f / sum;
    const long long r = row0 + row;
    __nv_bfloat16* dst = p.a.out + (tok0 + r / p.a.group) * p.a.o_tok + ((long long)kv_head * p.a.group + r % p.a.group) * p.a.o_head + d0;
    uint4 y = make_uint4(0, 0, 0, 0);
    if (any) y = make_uint4(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv),
                            pack_bf16x2(acc[4] * inv, acc[5] * inv), pack_bf16x2(acc[6] * inv, acc[7] * inv));
    *reinterpret_cast<uint4*>(dst) = y;
  }
}

}  // namespace sol
