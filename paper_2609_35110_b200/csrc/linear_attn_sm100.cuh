// Linear attention with a decay per head over the tokens of a plan, chunked form on tcgen05 tensor cores.
//
//   S_t = g S_{t-1} + k_t^T v_t,   o_t = scale * q_t S_t,   g = exp(log_decay[head])
//
// A tile of 128 tokens (positions i, j = 0..127 inside it, S the state before it, m the tokens it holds) gives
//   O     = P V + diag(g^{i+1}) Q S             P_ij = g^{i-j} <q_i, k_j> for j <= i, else 0
//   S'    = g^m S + K'^T V                      K'_j = g^{m-1-j} k_j
// four matrix products per tile instead of 128 steps, and only powers of g between 0 and m, which cannot overflow.
// A masked key, and a row behind the sequence's end, has P_ij = 0 and K'_j = 0.
//
// One CTA = one piece: seg_tiles consecutive tiles of one (sequence, head), walked in order with the state in fp32
// registers.  A sequence that is cut into several pieces takes two launches: the first (kStateOnly) computes, for every
// piece but the last, the state that the piece adds on its own; the second starts each piece from the sum of its
// predecessors' states (and the caller's), which it forms in a fixed order, and writes the outputs.  (One launch whose
// pieces hand their states on, so that the second walk finds K and V in L2, was built and measured: 1.6 to 2.0 ms where
// two launches take 1.4 ms at 111,856 tokens x 40 heads x 128.  What bounds the second walk is not HBM.)
//
// Precision: products of bf16 values are exact in the fp32 accumulators.  P and the copy of S that the tensor core reads
// are rounded to bf16 (they only enter bf16 outputs).  K' is split into two bf16 parts, hi + lo, so that the state, which
// is fp32 and carried from tile to tile, keeps about 16 bits of every factor instead of 8; the running state itself is
// never rounded below fp32 and never accumulated in tensor memory for longer than one tile.  The split needs three bf16x2
// instructions for two values: with the weight as w = wb + wc (two bf16), hi = rn(k wb), lo = rn(k wc + rn(k wb - hi)),
// where k wb - hi is exact before its rounding.  Every rounding is off by at most 2^-8 of its result: w - wb - wc is at most 2^-16
// of |w|, the rounded k wb - hi (2^-8 of |k w|) off by 2^-16 of |k w|, lo itself (2^-7 of |k w|) by 2^-15: 2^-14 of |k w| at
// worst, reached to more than a half (2.2 * 2^-16 for k = 1.0703125, w = 0.5292931), against 5 instructions for one value in fp32.
// Typically it is far less: measured, the state is within 4e-6 of fp64 in the 2-norm (fp32 arithmetic: 2.8e-7).  A third part would need 64 more columns of tensor
// memory, and fp16 parts (11 bits each) a V in fp16, whose range is narrower than what a caller may pass.
//
// Warp roles:
//   0-7    (A) two threads per query row: scores -> P (column blocks of 32 alternate between them), output epilogue
//   8-15   (B) K -> K', transposed on the way (ldmatrix) into tensor memory; two threads per K dim: a row of the state
//   16     TMA producer;   17  MMA issuer, owns the tensor memory;   18  TMA stores of the outputs
// (the state launch has no A and no stores: B is 0-7, 8 the producer, 9 the issuer).
// Tensor memory (512 columns): scores / P; K' hi | lo; the output, which is Q S first, scaled row by row by A, and then
// accumulates P V; K'^T V.  The state launch has no scores and no outputs: there K' and K'^T V alternate between two
// places, so that a tile is converted while its predecessor is multiplied.
//
// head_dim 64 (kPairs): a CTA serves two neighbouring heads at once.  Their Q, K and V side by side are tiles of 128 columns;
// K' and K'^T V are the products of a 128-dim head of which the two diagonal blocks count, and S is a block-diagonal matrix,
// so that Q S is one product too.  Only the scores and P V run per head, one after the other.  (One head per CTA left half of
// B and of the tensor-memory lanes idle: 0.58 ms for 38,871 tokens x 48 heads where pairs take 0.41 ms.)  With an odd number of
// heads the last pair's second head lies outside the tensors: its loads are filled with zeros, its stores are dropped.
//
// HBM needs 2.9 us per tile (4 x 128 x 128 x 2 bytes, every SM streaming).  What comes before it is shared-memory bandwidth,
// which operands of 128-wide products use up as fast as the tensor core, and with it the latency of everything that goes
// through that pipe, spilled registers included: so K' is a tensor-memory operand, outputs leave through the V tile's own
// space with a TMA store, nothing is staged twice, and the decay of a score is computed, not looked up.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include "device_types.cuh"
#include "ptx_sm100.cuh"
#include "step_kernels.cuh"

namespace sol {

struct LinearParams {
  const SeqDev* seqs;
  int n_seqs;
  int heads;
  int seg_tiles;              // tiles of a piece
  int n_cut;                  // sequences of more than one piece: the first ones of the schedule, which is longest first
  int cut_pieces;             // their pieces; then every sequence is one piece per unit
  const uint8_t* key_mask;    // uint8 [total_tokens] or nullptr
  const float* log_decay;     // [heads]
  float scale;
  const float* state_in;      // [n_seqs][heads][D][D] in the caller's order of sequences, or nullptr (zeros)
  float* state_out;           // the same, or nullptr
  float* local;               // states the pieces add on their own: [piece][D / 4][D rows] float4
  float* initial;             // copies of state_in, same layout: [sequence][head]
  __nv_bfloat16* out;
  long long o_tok_stride, o_head_stride;
  unsigned int* status;
  unsigned long long wait_limit_ns;
  unsigned int fault_inject;  // test hook: 1 = CTA 0 never publishes its first K'^T V (exercises the bounded waits)
};

// Bits i and i + 1 of a word -> mask of a pair of 16-bit values (without a branch).
__device__ __forceinline__ uint32_t pair_mask(uint32_t bits, int i) {
  const uint32_t lo = static_cast<uint32_t>(static_cast<int>(bits << (31 - i)) >> 31);
  const uint32_t hi = static_cast<uint32_t>(static_cast<int>(bits << (30 - i)) >> 31);
  return (lo & 0xffffu) | (hi & 0xffff0000u);
}

// Powers of the decay: log2(g) as the sum of two floats, so that the exponent of a high power keeps its low bits.
struct DecayPowers {
  float hi, lo;
  __device__ __forceinline__ explicit DecayPowers(float log_decay) {
    const double l = (log_decay > 0.f ? 0.0 : (double)log_decay) * 1.4426950408889634;      // NaN stays NaN
    hi = (float)l;
    lo = hi < -1e4f ? 0.f : (float)(l - (double)hi);
  }
  __device__ __forceinline__ float operator()(int d) const {
    if (d == 0) return 1.f;
    if (hi < -1e4f) return 0.f;                            // 2^-10000, and the -infinity that forgets everything
    const float x = (float)d * hi, e = fmaf((float)d, hi, -x) + (float)d * lo, r = exp2f(x);
    return fmaf(r, e * 0.6931471806f, r);
  }
};

// Main launch: 19 warps and an idle one, which completes a warpgroup; registers 640 threads x 96 = 256 x 88 + 256 x 128 + 128 x 48.
__host__ __device__ constexpr int linear_threads(bool state_only) { return state_only ? 320 : 640; }

template <bool kStateOnly>
struct LinearSmem {
  static constexpr int kTile = 128 * 128 * 2;                            // 128 tokens x 128 columns, two boxes of 64 columns
  static constexpr int kQStages = kStateOnly ? 0 : 2;
  static constexpr int kStages = kStateOnly ? 3 : 2;
  static constexpr int kOffQ = 0;
  static constexpr int kOffK = kOffQ + kQStages * kTile;
  static constexpr int kOffV = kOffK + kStages * kTile;
  static constexpr int kOffSt = kOffV + kStages * kTile;                 // bf16 copy of the state, laid out like V
  static constexpr int kOffTab = kOffSt + kTile;                         // per head: g^0 .. g^15, then g^0, g^16 .. g^128
  static constexpr int kOffPairs = kOffTab + 2 * 32 * 4;                  // per head: weights of the 64 token pairs of a whole tile, split
  static constexpr int kOffBars = kOffPairs + 2 * 64 * 8;
  static constexpr int kNumBars = 2 * kQStages + 5 * kStages + 11;
  static constexpr int kOffTmemPtr = kOffBars + kNumBars * 8;
  static constexpr int kBytes = kOffTmemPtr + 16;
  static constexpr int kDynBytes = kBytes + 1024;
  static_assert(kDynBytes <= 232448, "shared memory of one CTA");
};

// kPairs: head_dim 64, two heads per CTA; otherwise head_dim 128
template <bool kPairs, bool kStateOnly>
__global__ void __launch_bounds__(linear_threads(kStateOnly), 1)
linear_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o, const LinearParams p) {
  using L = LinearSmem<kStateOnly>;
  constexpr int D = kPairs ? 64 : 128, kHeads = kPairs ? 2 : 1;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t sbase = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - raw_addr);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kFirstB = kStateOnly ? 0 : 8, kTma = kFirstB + 8, kMma = kTma + 1, kStore = kTma + 2;

  const uint32_t sQ = sbase + L::kOffQ, sK = sbase + L::kOffK, sV = sbase + L::kOffV, sSt = sbase + L::kOffSt;
  const uint32_t bars = sbase + L::kOffBars;
  constexpr int kS = L::kStages, kQS = L::kQStages;
  auto bar_q_full = [&](int s) { return bars + 8u * s; };
  auto bar_q_empty = [&](int s) { return bars + 8u * (kQS + s); };
  auto bar_k_full = [&](int s) { return bars + 8u * (2 * kQS + s); };
  auto bar_k_empty = [&](int s) { return bars + 8u * (2 * kQS + kS + s); };
  auto bar_v_full = [&](int s) { return bars + 8u * (2 * kQS + 2 * kS + s); };
  auto bar_v_empty = [&](int s) { return bars + 8u * (2 * kQS + 3 * kS + s); };
  auto bar_o_staged = [&](int s) { return bars + 8u * (2 * kQS + 4 * kS + s); };
  constexpr int kSB = 2 * kQS + 5 * kS;
  auto bar_kp_full = [&](int t) { return bars + 8u * (kSB + (t & 1)); };
  auto bar_t_full = [&](int t) { return bars + 8u * (kSB + 2 + (t & 1)); };
  const uint32_t bar_st_full = bars + 8u * (kSB + 4), bar_qs_full = bars + 8u * (kSB + 5), bar_o_full = bars + 8u * (kSB + 6),
                 bar_o_empty = bars + 8u * (kSB + 7), bar_drain = bars + 8u * (kSB + 8), bar_s_full = bars + 8u * (kSB + 9),
                 bar_p_full = bars + 8u * (kSB + 10);
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(smem + L::kOffTmemPtr);
  float* tab = reinterpret_cast<float*>(smem + L::kOffTab);
  uint2* pairs = reinterpret_cast<uint2*>(smem + L::kOffPairs);

  // ---- which piece: sequences in schedule order, then segments, heads (or pairs) fastest: CTAs that run together read
  //      neighbouring heads of the same tokens.  The state-only launch leaves out each sequence's last segment.  Only the
  //      sequences that are cut are walked over (there are few: cutting is for filling SMs).
  const int units = (p.heads + kHeads - 1) / kHeads;
  int si = 0, first = 0, local_first = 0, n_seg = 1;
  if (!kStateOnly && (int)blockIdx.x >= p.cut_pieces) {
    const int whole = ((int)blockIdx.x - p.cut_pieces) / units;
    si = p.n_cut + whole;
    first = p.cut_pieces + whole * units;
  } else {
    for (;; ++si) {
      n_seg = (p.seqs[si].n_ktiles + p.seg_tiles - 1) / p.seg_tiles;
      const int here = (kStateOnly ? n_seg - 1 : n_seg) * units;
      if ((int)blockIdx.x < first + here || si + 1 >= p.n_cut) break;
      first += here;
      local_first += (n_seg - 1) * units;
    }
  }
  const int rel = (int)blockIdx.x - first;
  const int seg = rel / units, unit = rel - seg * units, head = unit * kHeads;              // head: the (first) one
  SOL_DEVICE_CHECK(p.status, si < p.n_seqs && rel >= 0 && seg < n_seg, kCheckWorkItem);
  const int n_tiles = min(p.seg_tiles, p.seqs[si].n_ktiles - seg * p.seg_tiles);
  const int tok0 = (int)p.seqs[si].tok_start + seg * p.seg_tiles * 128;     // first token of the piece in the packed tensors
  const int rem0 = p.seqs[si].n_tokens - seg * p.seg_tiles * 128;           // tokens from there to the sequence's end
  const unsigned long long limit = p.wait_limit_ns;

  if (warp == kTma && lane == 0) {
    for (int s = 0; s < kQS; ++s) { mbar_init(bar_q_full(s), 1); mbar_init(bar_q_empty(s), 1); }
    for (int s = 0; s < kS; ++s) {
      mbar_init(bar_k_full(s), 1); mbar_init(bar_k_empty(s), 1);
      mbar_init(bar_v_full(s), 1); mbar_init(bar_v_empty(s), 1);
      mbar_init(bar_o_staged(s), 8);
    }
    mbar_init(bar_s_full, 1);
    mbar_init(bar_p_full, 8);
    for (int t = 0; t < 2; ++t) { mbar_init(bar_kp_full(t), 8); mbar_init(bar_t_full(t), 1); }
    mbar_init(bar_qs_full, 1);
    mbar_init(bar_st_full, 8);
    mbar_init(bar_o_full, 1);
    mbar_init(bar_o_empty, 8);
    mbar_init(bar_drain, 1);
    fence_mbar_init();
    if (!kStateOnly) { prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_o); }
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  if (threadIdx.x == 0) tmem_ptr_smem[1] = *reinterpret_cast<volatile unsigned int*>(p.status);
  if (warp == kMma) { tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_ptr_smem)), 512); tmem_relinquish(); }
  auto powers_of = [&](int hd) { return DecayPowers(__ldg(p.log_decay + min(head + hd, p.heads - 1))); };
  auto split = [&](float w0, float w1) {                   // two weights as wb + wc, bf16x2 each
    const uint32_t wb = pack_bf16x2(w0, w1);
    return make_uint2(wb, pack_bf16x2(w0 - bf16_lo(wb), w1 - bf16_hi(wb)));
  };
  {
    const int hd = threadIdx.x >> 7, tid = threadIdx.x & 127;
    if (hd < kHeads) {
      const DecayPowers power = powers_of(hd);
      if (tid < 16) tab[32 * hd + tid] = power(tid);
      else if (tid < 25) tab[32 * hd + tid] = power(16 * (tid - 16));
      else if (tid >= 64) pairs[tid - 64 + 64 * hd] = split(power(127 - 2 * (tid - 64)), power(126 - 2 * (tid - 64)));
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_ptr_smem[0];
  if (tmem_ptr_smem[1] != 0) {                             // a fault recorded earlier stops later CTAs at the door
    __syncthreads();
    if (warp == kMma) tmem_dealloc(tmem_base, 512);
    return;
  }
  constexpr uint32_t kColS = 0, kColK = 128, kColO = 256, kColT = 384;     // kColK: K' hi [0,64), lo [64,128)
  // where K' and K'^T V of tile c go
  auto col_k = [&](int c) { return kStateOnly && (c & 1) ? kColS : kColK; };
  auto col_t = [&](int c) { return kStateOnly && (c & 1) ? kColO : kColT; };
  bool ok = true;

  if (warp < kFirstB) {
    // =========================================================== A: scores -> P, outputs; two threads per query row
    if constexpr (!kStateOnly) {
    setmaxnreg_dec<88>();
    const int wq = warp & 3, half = warp >> 2;
    const int row = wq * 32 + lane;
    const uint32_t tm = tmem_base + (static_cast<uint32_t>(wq * 32) << 16);
    {
      // The decay of a score, scale * g^{row - j}, without a table (shared memory is what this kernel is short of).  The
      // exponent is the integer distance times log2(g), so that it is exactly 0 on the diagonal whatever log2(g) is: walked
      // along the columns in steps of log2(g), what was left there of cancelling numbers put a token's own weight off by up
      // to 3 % under strong decays.  From log2(g) = -256 on only the diagonal counts (2^-256 is 0 in fp32), and -infinity * 0
      // would be NaN: hence the limit.  Columns above the diagonal get whatever comes out and are masked.  All loops over columns
      // are rolled: unrolled, the five roles' code did not fit the instruction cache, and waiting for instructions was the
      // largest stall.
      auto log2_decay = [&](int hd) {
        const float l2 = powers_of(hd).hi;
        return l2 < -256.f ? -256.f : l2;                                  // (fmaxf would lose a NaN)
      };
      const float l2s[2] = {log2_decay(0), kPairs ? log2_decay(1) : 0.f};
      const float g1 = p.scale * powers_of(kPairs ? half : 0)(row + 1);    // this thread's 64 columns are one head's
      const float2 g1_2 = make_float2(g1, g1);
      const float2 scale2 = make_float2(p.scale, p.scale);

      auto make_p = [&](int c, int hd) {                                   // P of tile c, head hd
        const int m = min(128, rem0 - c * 128);
        const bool mixed = p.key_mask != nullptr || m < 128;
        uint32_t bits[2] = {~0u, ~0u};                                     // of this thread's two column blocks
        if (mixed) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int j = 32 * (2 * b + half) + lane;
            bool valid = j < m;
            if (valid && p.key_mask != nullptr) valid = p.key_mask[(long long)tok0 + c * 128 + j] != 0;
            bits[b] = __ballot_sync(0xffffffffu, valid);
          }
        }
        const float l2 = hd ? l2s[1] : l2s[0];
        ok = __all_sync(0xffffffffu, mbar_wait(bar_s_full, (c * kHeads + hd) & 1, limit));
        if (!ok) return;
        tc_fence_after();
        // P of 16 columns replaces the scores of a block of 32, in its first 16 columns (two chunks of 8): a block is read
        // and written by one warp alone, its second half before the first is overwritten.  Blocks right of the diagonal are zero.
#pragma unroll 1
        for (int b = 0; b < 2; ++b) {
          const int cb = 2 * b + half;
          const uint32_t at = tm + kColS + cb * 32;
          const int last = row - cb * 32;                                  // columns up to here lie left of the diagonal or on it
          const uint32_t on = (b ? bits[1] : bits[0]) & (last >= 31 ? ~0u : last < 0 ? 0u : (2u << last) - 1u);
          uint32_t s[32];
          if (cb <= wq) {
            tmem_ld32(at, s);
            tmem_wait_ld();
          }
          uint32_t pk[16];
          float2 dist = make_float2((float)last, (float)(last - 1));       // row - j of two columns
          const float2 l2_2 = make_float2(l2, l2), minus2 = make_float2(-2.f, -2.f);
          if (cb <= wq) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float2 x = mul_f32x2(l2_2, dist);
              const float2 w = mul_f32x2(scale2, make_float2(ex2_approx(x.x), ex2_approx(x.y)));
              const float2 y = mul_f32x2(make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), w);
              pk[e] = pack_bf16x2(y.x, y.y);
              dist = add_f32x2(dist, minus2);
            }
            if (cb == wq || mixed) {
#pragma unroll
              for (int e = 0; e < 16; ++e) pk[e] &= pair_mask(on, 2 * e);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) pk[e] = 0u;
          }
          tmem_st16(at, pk);
        }
      };
      auto p_done = [&]() {                                                // P (and the scaled Q S) are in place
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p_full);
      };
      // Q S of tile c times g^{i+1}, in place: P V is then accumulated on top
      auto scale_qs = [&](int c) {
        ok = __all_sync(0xffffffffu, mbar_wait(bar_qs_full, c & 1, limit));
        if (!ok) return;
        tc_fence_after();
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
          const uint32_t at = tm + kColO + half * 64 + i * 16;
          uint32_t a[16];
          tmem_ld16(at, a);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float2 x = mul_f32x2(g1_2, make_float2(__uint_as_float(a[e]), __uint_as_float(a[e + 1])));
            a[e] = __float_as_uint(x.x);
            a[e + 1] = __float_as_uint(x.y);
          }
          tmem_st16(at, a);
        }
      };

#pragma unroll 1
      for (int c = 0; c < n_tiles && ok; ++c) {
#pragma unroll 1
        for (int hd = 0; hd < kHeads && ok; ++hd) {
          make_p(c, hd);
          if (ok && hd == 0) scale_qs(c);
          if (ok) p_done();
        }
        if (!ok) break;
        const int m = min(128, rem0 - c * 128);
        ok = __all_sync(0xffffffffu, mbar_wait(bar_o_full, c & 1, limit));
        if (!ok) break;
        tc_fence_after();
        // The rows are staged where the tile's V was (nothing reads it any more), in the layout the TMA store expects.  A
        // tile that reaches beyond its sequence is written row by row instead: the rows behind it are not ours.
        const int stage_n = c % kS;
        uint8_t* stage = smem + L::kOffV + stage_n * L::kTile;
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {                          // 32 of this thread's 64 columns
          const int at0 = half * 8 + i * 4;             // first of their four 16-byte chunks of the row
          uint32_t a[32];
          tmem_ld32(tm + kColO + at0 * 8, a);
          tmem_wait_ld();
          if (i == 1) {                               // everything is in registers: the accumulators are free
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_o_empty);
          }
          uint4 w[4];
#pragma unroll
          for (int ch = 0; ch < 4; ++ch)
            w[ch] = make_uint4(pack_bf16x2(__uint_as_float(a[8 * ch]), __uint_as_float(a[8 * ch + 1])),
                               pack_bf16x2(__uint_as_float(a[8 * ch + 2]), __uint_as_float(a[8 * ch + 3])),
                               pack_bf16x2(__uint_as_float(a[8 * ch + 4]), __uint_as_float(a[8 * ch + 5])),
                               pack_bf16x2(__uint_as_float(a[8 * ch + 6]), __uint_as_float(a[8 * ch + 7])));
          if (m == 128) {
            uint8_t* to = stage + (at0 >> 3) * 16384 + row * 128;
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) *reinterpret_cast<uint4*>(to + ((((at0 & 7) + ch) ^ (row & 7)) << 4)) = w[ch];
          } else if (row < m && (!kPairs || head + half < p.heads)) {
            __nv_bfloat16* to = p.out + ((long long)tok0 + c * 128 + row) * p.o_tok_stride +
                                (long long)(kPairs ? head + half : head) * p.o_head_stride + (kPairs ? at0 & 7 : at0) * 8;
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) *reinterpret_cast<uint4*>(to + ch * 8) = w[ch];
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_o_staged(stage_n));
      }
    }
    if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutSoftmax);
    }
  } else if (warp < kTma) {
    // =========================================================== B: K -> K', state; two threads per token row / K dim
    if (!kStateOnly) setmaxnreg_inc<128>();
    const int wq = (warp - kFirstB) & 3, half = (warp - kFirstB) >> 2;
    const int row = wq * 32 + lane;
    constexpr int kCols = D / 2;                                           // columns of this thread's part of a row
    const int hd = kPairs ? wq >> 1 : 0, col0 = (kPairs ? 64 * hd : 0) + half * kCols;  // the row's head, its part's first column
    const bool has_state = head + hd < p.heads;                            // warp-uniform
    const uint32_t tm = tmem_base + (static_cast<uint32_t>(wq * 32) << 16) + col0;
    float S[kCols];
    // where this thread's 16-byte chunks of a row are in a tile (128-byte swizzle); D = 128: half = 64-column box
    auto chunk = [&](int r7, int ch) {
      const int at = col0 / 8 + ch;
      return (at >> 3) * 16384 + row * 128 + (((at & 7) ^ r7) << 4);
    };
    // row & 7, anew for every use: the compiler would otherwise keep all chunk addresses in registers throughout
    auto row7 = [&]() {
      int r7 = row & 7;
      asm volatile("" : "+r"(r7));
      return r7;
    };
    auto publish = [&]() {
      // this part of the state's row, rounded to bf16, in the layout of a V tile (row = contraction index)
      const int r7 = row7();
#pragma unroll
      for (int ch = 0; ch < kCols / 8; ++ch) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = S[ch * 8 + e];
        *reinterpret_cast<uint4*>(smem + L::kOffSt + chunk(r7, ch)) = pack8(f);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_st_full);
    };
    // K' of this warp: K dims 32 wq .. + 31 (tensor-memory lanes), tokens 64 half .. + 63.  ldmatrix hands thread i the token
    // pairs 64 half + 8 t + 2 (i % 4), + 1 for t = 0..7.  The weights wb + wc of a pair of tokens of a whole tile are two
    // words of a table; other tiles compute them.
    auto weight = [&](int e) { return e < 0 ? 0.f : tab[32 * hd + (e & 15)] * tab[32 * hd + 16 + (e >> 4)]; };       // g^e
    // address of this lane's row for ldmatrix: lanes 0-7 and 16-23 the first 8 of 16 dims, the others the second 8; lanes
    // 0-15 the first of two token blocks, the others the second
    const uint32_t k_row = (64 * half + ((lane >> 4) << 3) + (lane & 7)) * 128;
    const int dc_in = (lane >> 3) & 1;

    // K' of tile n of the ring, into tensor memory at col; rem: tokens from the tile's first one to the sequence's end
    auto convert = [&](int n, int rem, uint32_t col) {
      const int m = min(128, rem);
      const bool mixed = p.key_mask != nullptr || m < 128;
      const int st = n % kS;
      const uint32_t ph = (n / kS) & 1;
      uint32_t bits_lo = ~0u, bits_hi = ~0u, vbits = ~0u;                  // tokens 64 half .., + 32 ..; token rows 32 wq ..
      if (mixed) {
#pragma unroll
        for (int b = 0; b < 3; ++b) {
          const int j = (b < 2 ? 64 * half + 32 * b : 32 * wq) + lane;
          bool valid = j < m;
          if (valid && p.key_mask != nullptr) valid = p.key_mask[(long long)tok0 + n * 128 + j] != 0;
          const uint32_t word = __ballot_sync(0xffffffffu, valid);
          if (b == 0) bits_lo = word; else if (b == 1) bits_hi = word; else vbits = word;
        }
      }
      ok = __all_sync(0xffffffffu, mbar_wait(bar_k_full(st), ph, limit));
      if (!ok) return;
      tc_fence_after();
#pragma unroll 1
        for (int tg = 0; tg < 2; ++tg) {                                   // 32 tokens
          uint2 w[4];                                                      // of this thread's pairs in the four token blocks
          uint32_t on[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int in = 32 * tg + 8 * t + 2 * (lane & 3);               // the pair's first token, from token 64 half on
            if (!mixed) {
              w[t] = pairs[64 * hd + 32 * half + (in >> 1)];
              on[t] = ~0u;
            } else {
              const int e = m - 1 - (64 * half + in);
              w[t] = split(weight(e), weight(e - 1));
              on[t] = pair_mask(tg ? bits_hi : bits_lo, in & 31);
            }
          }
#pragma unroll
          for (int lh = 0; lh < 2; ++lh) {                                 // 16 of the 32 K dims
            const int dc = 4 * wq + 2 * lh + dc_in;                        // 16-byte chunk of the row
            const uint32_t src = sK + st * L::kTile + (dc >> 3) * 16384 + k_row + (((dc & 7) ^ (lane & 7)) << 4);
            uint32_t x[2][4];
            ldmatrix_x4_trans(src + tg * 32 * 128, x[0]);
            ldmatrix_x4_trans(src + tg * 32 * 128 + 16 * 128, x[1]);
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {                                  // token block r / 2
              const uint32_t k2 = x[r >> 2][r & 3] & on[r >> 1];           // whatever stands under a mask, NaN included, is dropped
              hi[r] = mul_bf16x2(k2, w[r >> 1].x);
              lo[r] = fma_bf16x2(k2, w[r >> 1].y, fma_bf16x2(k2, w[r >> 1].x, hi[r] ^ 0x80008000u));
            }
            const uint32_t dst = tmem_base + (static_cast<uint32_t>(wq * 32 + lh * 16) << 16) + col + half * 32 + tg * 16;
            tmem_st_16x128b_x4(dst, hi);
            tmem_st_16x128b_x4(dst + 64, lo);
          }
        }
        tmem_wait_st();
      if (mixed) {
        // V rows that do not count become zeros: 0 * (whatever stands there) would not be 0 for infinities and NaN
        ok = __all_sync(0xffffffffu, mbar_wait(bar_v_full(st), ph, limit));
        if (!ok) return;
        if (((vbits >> lane) & 1u) == 0) {                                 // box `half` of token row `row`
#pragma unroll
          for (int ch = 0; ch < 8; ++ch)
            *reinterpret_cast<uint4*>(smem + L::kOffV + st * L::kTile + half * 16384 + row * 128 + ch * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_kp_full(n));
    };
    // S = g^m S + K'^T V of tile n, read from col
    auto update = [&](int n, int rem, uint32_t col) {
      const int m = min(128, rem);
      ok = __all_sync(0xffffffffu, mbar_wait(bar_t_full(n), (n >> 1) & 1, limit));
      if (!ok) return;
      tc_fence_after();
        const float gm = weight(m);
#pragma unroll
        for (int cb = 0; cb < kCols / 16; ++cb) {
          uint32_t t[16];
          tmem_ld16(tm + col + cb * 16, t);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float2 x = fma_f32x2(make_float2(gm, gm), make_float2(S[cb * 16 + e], S[cb * 16 + e + 1]),
                                       make_float2(__uint_as_float(t[e]), __uint_as_float(t[e + 1])));
            S[cb * 16 + e] = x.x;
            S[cb * 16 + e + 1] = x.y;
          }
        }
        tc_fence_before();
    };

#pragma unroll
    for (int e = 0; e < kCols; ++e) S[e] = 0.f;
    // the state before this piece
    auto add_piece = [&](const float* piece, float g) {                    // S = g S + what a piece left in the workspace
      const float4* src = reinterpret_cast<const float4*>(piece) + half * (kCols / 4) * 128 + row;
#pragma unroll
      for (int e = 0; e < kCols / 4; ++e) {
        const float4 x = src[e * 128];
        S[4 * e] = fmaf(g, S[4 * e], x.x); S[4 * e + 1] = fmaf(g, S[4 * e + 1], x.y);
        S[4 * e + 2] = fmaf(g, S[4 * e + 2], x.z); S[4 * e + 3] = fmaf(g, S[4 * e + 3], x.w);
      }
    };
    auto leave_piece = [&](float* piece) {
      float4* dst = reinterpret_cast<float4*>(piece) + half * (kCols / 4) * 128 + row;
#pragma unroll
      for (int e = 0; e < kCols / 4; ++e) dst[e * 128] = make_float4(S[4 * e], S[4 * e + 1], S[4 * e + 2], S[4 * e + 3]);
    };
    // The caller's states have rows of D values.  A thread reading its own row would touch 32 lines per instruction, so a warp
    // moves 32 rows x 32 columns at a time, eight lanes per row, through 4 KB of its own in the place of the bf16 copy.
    uint8_t* mine = smem + L::kOffSt + (warp - kFirstB) * 4096;
    const long long state0 = (((long long)p.seqs[si].seq_id * p.heads + head + hd) * D + (row - lane) % D) * D + half * kCols;
    const int l8 = lane & 7, r4 = lane >> 3;
    auto read_state = [&](const float* state) {
#pragma unroll
      for (int b = 0; b < kCols / 32; ++b) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<float4*>(mine + (4 * i + r4) * 128 + ((l8 ^ ((4 * i + r4) & 7)) << 4)) =
              *reinterpret_cast<const float4*>(state + state0 + (4 * i + r4) * D + b * 32 + l8 * 4);
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float4 x = *reinterpret_cast<const float4*>(mine + lane * 128 + ((e ^ l8) << 4));
          S[b * 32 + 4 * e] = x.x; S[b * 32 + 4 * e + 1] = x.y; S[b * 32 + 4 * e + 2] = x.z; S[b * 32 + 4 * e + 3] = x.w;
        }
        __syncwarp();
      }
    };
    auto write_state = [&](float* state) {
#pragma unroll
      for (int b = 0; b < kCols / 32; ++b) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          *reinterpret_cast<float4*>(mine + lane * 128 + ((e ^ l8) << 4)) =
              make_float4(S[b * 32 + 4 * e], S[b * 32 + 4 * e + 1], S[b * 32 + 4 * e + 2], S[b * 32 + 4 * e + 3]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<float4*>(state + state0 + (4 * i + r4) * D + b * 32 + l8 * 4) =
              *reinterpret_cast<const float4*>(mine + (4 * i + r4) * 128 + ((l8 ^ ((4 * i + r4) & 7)) << 4));
        __syncwarp();
      }
    };
    if (seg == 0 && p.state_in != nullptr) {
      // A cut sequence: the state launch is the only one that reads state_in (its first piece starts from it and leaves a
      // copy), so that the main launch may write state_out to the same memory at any time.
      float* copy = p.initial + (long long)(si * units + unit) * (128 * D);
      if (kStateOnly || n_seg == 1) {
        // a decay of 0 forgets whatever the state holds, infinities and NaN included: 0 * S would not
        if (has_state && weight(1) != 0.f) read_state(p.state_in);
        asm volatile("bar.sync 1, 256;" ::: "memory");                     // the others' staging space is theirs until here
        if (kStateOnly) leave_piece(copy);
      } else {
        add_piece(copy, 0.f);
      }
    }
    if constexpr (!kStateOnly) {
      if (kPairs) {                                                        // S beside its diagonal blocks: this row's half of it
#pragma unroll
        for (int ch = 0; ch < 4; ++ch)
          *reinterpret_cast<uint4*>(smem + L::kOffSt + (hd ^ 1) * 16384 + row * 128 + half * 64 + ch * 16) = make_uint4(0, 0, 0, 0);
      }
      if (seg > 0) {
        const float gs = powers_of(hd)(128 * p.seg_tiles);                 // every earlier segment is whole
        for (int r = 0; r < seg; ++r) add_piece(p.local + (long long)(local_first + r * units + unit) * (128 * D), gs);
      }
      publish();
    }
    // the state launch converts one tile ahead
    constexpr int kAhead = kStateOnly ? 1 : 0;
#pragma unroll 1
    for (int c = 0; c < n_tiles + kAhead; ++c) {
      if (c < n_tiles) convert(c, rem0 - c * 128, col_k(c));
      if (!ok) break;
      if (c < kAhead) continue;
      update(c - kAhead, rem0 - (c - kAhead) * 128, col_t(c - kAhead));
      if (!ok) break;
      if (!kStateOnly && c + 1 < n_tiles) publish();
    }
    if (ok) {
      if constexpr (kStateOnly) {
        leave_piece(p.local + (long long)(local_first + rel) * (128 * D));
      } else if (has_state && seg == n_seg - 1 && p.state_out != nullptr) {
        write_state(p.state_out);
      }
    }
    if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutSoftmax);
  } else if (!kStateOnly) {
    setmaxnreg_dec<48>();
  }

  if (warp == kTma) {
    // =========================================================== TMA producer
    if (lane == 0) {
      const uint64_t pol_once = l2_policy_evict_first();
      auto load = [&](const CUtensorMap* tm, uint32_t base, uint32_t full, int st, int tok, bool once) {
        mbar_arrive_expect_tx(full, L::kTile);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int x = kPairs ? 0 : hf * 64, h = kPairs ? head + hf : head;
          if (once) tma_load_3d_hint(base + st * L::kTile + hf * 16384, tm, full, x, h, tok, pol_once);
          else      tma_load_3d(base + st * L::kTile + hf * 16384, tm, full, x, h, tok);
        }
      };
      int c = 0;
      for (; c < n_tiles; ++c) {
        const int st = c % kS, tok = tok0 + c * 128;
        const uint32_t par = ((c / kS) & 1) ^ 1u;
        if (!mbar_wait(bar_k_empty(st), par, limit)) { ok = false; break; }
        load(&tm_k, sK, bar_k_full(st), st, tok, false);
        if constexpr (!kStateOnly) {
          const int qs = c % kQS;
          if (!mbar_wait(bar_q_empty(qs), ((c / kQS) & 1) ^ 1u, limit)) { ok = false; break; }
          load(&tm_q, sQ, bar_q_full(qs), qs, tok, true);
        }
        if (!mbar_wait(bar_v_empty(st), par, limit)) { ok = false; break; }
        load(&tm_v, sV, bar_v_full(st), st, tok, false);
      }
      if (!ok) {
        atomicCAS(p.status, 0u, kStatusTimeoutProducer);
        // copies still in flight land before the shared memory is given back; the latest ones (K and Q of the tile it gave
        // up in) take far less than the limit that has just run out
        for (int b = max(0, c - kS); b < c; ++b) {
          mbar_wait(bar_k_full(b % kS), (b / kS) & 1, limit);
          mbar_wait(bar_v_full(b % kS), (b / kS) & 1, limit);
        }
      }
    }
    __syncwarp();
  } else if (warp == kMma) {
    // =========================================================== MMA issuer
    constexpr uint32_t idesc_qk = idesc_bf16_f32(128, 128, false);
    constexpr uint32_t idesc_d = idesc_bf16_f32(128, 128, true);           // B MN-major: Q S and K'^T V
    constexpr uint32_t idesc_pv = idesc_bf16_f32(128, D, true);            // P V of one head
    const uint32_t hi_desc = smem_desc_hi_sw128(1024);
    const uint32_t q_lo = smem_desc_lo(sQ, 16), k_lo = smem_desc_lo(sK, 16);
    const uint32_t v_lo = smem_desc_lo(sV, 16384), st_lo = smem_desc_lo(sSt, 16384);
    constexpr uint32_t kStep = L::kTile >> 4;
    auto wait = [&](uint32_t bar, uint32_t parity) { return ok = mbar_wait_warp(bar, parity, limit); };
    // scores of tile n, head hd (the P V that read P in the same place was issued before)
    auto issue_scores = [&](int n, int hd) {
      const int qs = n % max(kQS, 1), st = n % kS;
      if (hd == 0 && (!wait(bar_k_full(st), (n / kS) & 1) || !wait(bar_q_full(qs), (n / max(kQS, 1)) & 1))) return;
      tc_fence_after();
#pragma unroll 1
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t off = ((hd + (k >> 2)) * 16384 + (k & 3) * 32) >> 4;
        mma_ss_elect<false>(tmem_base + kColS, q_lo + qs * kStep + off, k_lo + st * kStep + off, hi_desc, idesc_qk, k);
      }
      tc_commit_elect(bar_s_full);
    };
    // what tile kt adds to the state; the product that was there before has been read when K' is ready
    auto issue_state = [&](int kt) {
      const uint32_t from = col_k(kt), to = col_t(kt);
      const int st = kt % kS;
      if (!wait(bar_v_full(st), (kt / kS) & 1) || !wait(bar_kp_full(kt), (kt >> 1) & 1)) return;
      tc_fence_after();
#pragma unroll 1
      for (int k = 0; k < 16; ++k)                                         // hi, then lo
        mma_ts_elect<false>(tmem_base + to, tmem_base + from + k * 8, v_lo + st * kStep + (k & 7) * (2048 >> 4), hi_desc, idesc_d, k);
      if (!(p.fault_inject == 1u && blockIdx.x == 0 && kt == 0)) tc_commit_elect(bar_t_full(kt));
      if (!kPairs || kStateOnly) tc_commit_elect(bar_k_empty(st));         // (pairs: the second head's scores need K still)
    };
    if constexpr (kStateOnly) {
      for (int c = 0; c < n_tiles; ++c) {
        issue_state(c);
        if (!ok) break;
        tc_commit_elect(bar_v_empty(c % kS));
      }
    } else {
      issue_scores(0, 0);
      for (int c = 0; c < n_tiles && ok; ++c) {
        const int st = c % kS, qs = c % kQS;
        // Q times the state before this tile
        if (!wait(bar_st_full, c & 1)) break;
        if (c > 0 && !wait(bar_o_empty, (c - 1) & 1)) break;
        tc_fence_after();
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
          const uint32_t off = ((k >> 2) * 16384 + (k & 3) * 32) >> 4;
          mma_ss_elect<false>(tmem_base + kColO, q_lo + qs * kStep + off, st_lo + k * (2048 >> 4), hi_desc, idesc_d, k);
        }
        tc_commit_elect(bar_qs_full);
        if (!kPairs) tc_commit_elect(bar_q_empty(qs));
        issue_state(c);
        if (!ok) break;
#pragma unroll 1
        for (int hd = 0; hd < kHeads; ++hd) {
          if (!wait(bar_p_full, (c * kHeads + hd) & 1)) break;
          tc_fence_after();
#pragma unroll 1
          for (int k = 0; k < 8; ++k)                                      // on top of the scaled Q S
            mma_ts_elect<true>(tmem_base + kColO + hd * 64, tmem_base + kColS + (k >> 1) * 32 + (k & 1) * 8,
                               v_lo + st * kStep + ((hd * 16384 + k * 2048) >> 4), hi_desc, idesc_pv, 1u);
          if (hd + 1 < kHeads) {
            issue_scores(c, hd + 1);
            if (!ok) break;
            tc_commit_elect(bar_q_empty(qs));
            tc_commit_elect(bar_k_empty(st));
          }
        }
        if (!ok) break;
        tc_commit_elect(bar_o_full);                                       // (V's space is released once the outputs staged there are out)
        if (c + 1 < n_tiles) issue_scores(c + 1, 0);
      }
    }
    if (!ok) {
      if (lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutMma);
      tc_commit_elect(bar_drain);
      mbar_wait_warp(bar_drain, 0, limit);
    }
    __syncwarp();
  } else if (warp == kStore) {
    // =========================================================== output stores
    if constexpr (!kStateOnly) {
      if (lane == 0) {
        for (int c = 0; c < n_tiles; ++c) {
          const int st = c % kS;
          if (!mbar_wait(bar_o_staged(st), (c / kS) & 1, limit)) { atomicCAS(p.status, 0u, kStatusTimeoutSoftmax); break; }
          if (rem0 - c * 128 >= 128) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
              if (!kPairs || head + hf < p.heads)
                tma_store_3d(&tm_o, sV + st * L::kTile + hf * 16384, kPairs ? 0 : hf * 64, kPairs ? head + hf : head, tok0 + c * 128);
            bulk_commit_group();
            bulk_wait_read_all();
          }
          mbar_arrive(bar_v_empty(st));
        }
      }
    }
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kMma) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

}  // namespace sol
