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
// predecessors' states (and the caller's), which it forms in a fixed order, and writes the outputs.
//
// Precision: products of bf16 values are exact in the fp32 accumulators.  P and the copy of S that the tensor core reads
// are rounded to bf16 (they only enter bf16 outputs).  K' is split into two bf16 parts, hi + lo, so that the state, which
// is fp32 and carried from tile to tile, keeps about 16 bits of every factor instead of 8; the running state itself is
// never rounded below fp32 and never accumulated in tensor memory for longer than one tile.  The split needs three bf16x2
// instructions for two values: with the weight as w = wb + wc (two bf16), hi = rn(k wb), lo = rn(k wc + rn(k wb - hi)),
// where k wb - hi is exact before its rounding.  That is off by at most 2^-16 of |k w| (half a step, 2^-8, of two
// quantities that are themselves at most 2^-8 of it, and of wc), against 5 instructions for one value in fp32.
//
// Warp roles (the state launch has only the second group, the producer and the issuer):
//   8 warps   two threads per query row: scores -> P (column blocks of 32 alternate between them), output epilogue
//   8 warps   K -> K', transposed on the way (ldmatrix) into tensor memory; two threads per K dim: a row of the state
//   1 warp    TMA producer;   1 warp: MMA issuer, owns the tensor memory;   1 warp: TMA stores of the outputs
// Tensor memory (512 columns): scores / P [0,128); K' hi | lo [128,256), replaced by P V; Q S [256,384); K'^T V [384,512).
//
// Bound by HBM: 4 x 128 x D x 2 bytes per tile and head (2.9 us at D = 128 with every SM streaming) against 5 small
// products (4 and the lo half).  Next comes shared-memory bandwidth, which operands of 128-wide products use up as fast as
// the tensor core: so K' is a tensor-memory operand, outputs leave through the V tile's own space with a TMA store, and
// nothing is staged twice.
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
};

// Compute warps, then the producer, the MMA issuer and (main launch) the store warp and an idle one, which completes a
// warpgroup.  Registers of the main launch: 640 threads x 96 = 256 x 88 + 256 x 128 + 128 x 48.
constexpr int linear_threads(bool state_only) { return state_only ? 320 : 640; }

template <int D, bool kStateOnly>
struct LinearSmem {
  static constexpr int kTile = 128 * D * 2;
  static constexpr int kHalves = D / 64;
  static constexpr int kQStages = kStateOnly ? 0 : 2;
  static constexpr int kStages = D == 128 ? (kStateOnly ? 3 : 2) : 4;
  static constexpr int kOffQ = 0;
  static constexpr int kOffK = kOffQ + kQStages * kTile;
  static constexpr int kOffV = kOffK + kStages * kTile;
  static constexpr int kOffSt = kOffV + kStages * kTile;                 // bf16 copy of the state, laid out like V
  static constexpr int kOffDec = kOffSt + (kStateOnly ? 0 : D * D * 2);  // powers of the decay: [128 + d], zero for d < 0
  static constexpr int kOffFall = kOffDec + 260 * 4;                     // g^31 .. g^0
  static constexpr int kOffBars = kOffFall + 32 * 4;
  static constexpr int kNumBars = 2 * kQStages + 4 * kStages + 9;
  static constexpr int kOffTmemPtr = kOffBars + kNumBars * 8;
  static constexpr int kBytes = kOffTmemPtr + 16;
  static constexpr int kDynBytes = kBytes + 1024;
};

template <int D, bool kStateOnly>
__global__ void __launch_bounds__(linear_threads(kStateOnly), 1)
linear_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o, const LinearParams p) {
  using L = LinearSmem<D, kStateOnly>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t sbase = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - raw_addr);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kFirstB = kStateOnly ? 0 : 8, kTma = kFirstB + 8, kMma = kTma + 1, kStore = kTma + 2;

  const uint32_t sQ = sbase + L::kOffQ, sK = sbase + L::kOffK, sV = sbase + L::kOffV, sSt = sbase + L::kOffSt;
  float* dec = reinterpret_cast<float*>(smem + L::kOffDec) + 128;       // dec[d] = g^d, d in [-128, 128]
  const uint32_t bars = sbase + L::kOffBars;
  constexpr int kQB = 2 * L::kQStages, kSB = kQB + 4 * L::kStages;
  auto bar_q_full = [&](int s) { return bars + 8u * s; };
  auto bar_q_empty = [&](int s) { return bars + 8u * (L::kQStages + s); };
  auto bar_k_full = [&](int s) { return bars + 8u * (kQB + s); };
  auto bar_k_empty = [&](int s) { return bars + 8u * (kQB + L::kStages + s); };
  auto bar_v_full = [&](int s) { return bars + 8u * (kQB + 2 * L::kStages + s); };
  auto bar_v_empty = [&](int s) { return bars + 8u * (kQB + 3 * L::kStages + s); };
  const uint32_t bar_s_full = bars + 8u * (kSB + 0), bar_p_full = bars + 8u * (kSB + 1), bar_kp_full = bars + 8u * (kSB + 2),
                 bar_t_full = bars + 8u * (kSB + 3), bar_st_full = bars + 8u * (kSB + 4), bar_o_full = bars + 8u * (kSB + 5),
                 bar_o_empty = bars + 8u * (kSB + 6), bar_o_staged = bars + 8u * (kSB + 7), bar_drain = bars + 8u * (kSB + 8);
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(smem + L::kOffTmemPtr);

  // ---- which piece: sequences in schedule order, then segments, heads fastest (CTAs that run together read neighbouring
  //      heads of the same tokens).  The state-only launch leaves out each sequence's last segment.
  int si = 0, first = 0, local_first = 0, n_seg = 0;
  for (;; ++si) {
    n_seg = (p.seqs[si].n_ktiles + p.seg_tiles - 1) / p.seg_tiles;
    const int here = (kStateOnly ? n_seg - 1 : n_seg) * p.heads;
    if ((int)blockIdx.x < first + here || si + 1 >= p.n_seqs) break;
    first += here;
    local_first += (n_seg - 1) * p.heads;
  }
  const SeqDev sq = p.seqs[si];
  const int rel = (int)blockIdx.x - first;
  const int seg = rel / p.heads, head = rel - seg * p.heads;
  SOL_DEVICE_CHECK(p.status, rel >= 0 && seg < n_seg, kCheckWorkItem);
  const int tile0 = seg * p.seg_tiles;
  const int n_tiles = min(p.seg_tiles, sq.n_ktiles - tile0);
  const unsigned long long limit = p.wait_limit_ns;
  const int tok0 = (int)sq.tok_start;

  if (warp == kTma && lane == 0) {
    for (int s = 0; s < L::kQStages; ++s) { mbar_init(bar_q_full(s), 1); mbar_init(bar_q_empty(s), 1); }
    for (int s = 0; s < L::kStages; ++s) {
      mbar_init(bar_k_full(s), 1); mbar_init(bar_k_empty(s), 1);
      mbar_init(bar_v_full(s), 1); mbar_init(bar_v_empty(s), 1);
    }
    mbar_init(bar_s_full, 1);
    mbar_init(bar_p_full, 8);
    mbar_init(bar_kp_full, 8);
    mbar_init(bar_t_full, 1);
    mbar_init(bar_st_full, 8);
    mbar_init(bar_o_full, 1);
    mbar_init(bar_o_empty, 8);
    mbar_init(bar_o_staged, 8);
    mbar_init(bar_drain, 1);
    fence_mbar_init();
    if (!kStateOnly) { prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_o); }
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  if (threadIdx.x == 0) tmem_ptr_smem[1] = *reinterpret_cast<volatile unsigned int*>(p.status);
  if (warp == kMma) { tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_ptr_smem)), 512); tmem_relinquish(); }
  const double ld = fmin((double)__ldg(p.log_decay + head), 0.0);
  if (threadIdx.x < 257) {
    const int d = (int)threadIdx.x - 128;
    dec[d] = d < 0 ? 0.f : d == 0 ? 1.f : (float)exp((double)d * ld);     // (0 * -inf is NaN: g^0 is 1)
  }
  float4* fall = reinterpret_cast<float4*>(smem + L::kOffFall);
  if (threadIdx.x >= 288 && threadIdx.x < 320) {
    const int d = 319 - (int)threadIdx.x;
    reinterpret_cast<float*>(fall)[31 - d] = d == 0 ? 1.f : (float)exp((double)d * ld);
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
  constexpr uint32_t kColS = 0, kColO = 128, kColQS = 256, kColT = 384;

  if (warp < kFirstB) {
    if constexpr (!kStateOnly) {
      // =========================================================== scores -> P, outputs; two threads per query row
      setmaxnreg_dec<88>();
      const int wq = warp & 3, half = warp >> 2;
      const int row = wq * 32 + lane;
      const uint32_t tm = tmem_base + (static_cast<uint32_t>(wq * 32) << 16);
      const float g1 = p.scale * dec[row + 1];
      const float2 g1_2 = make_float2(g1, g1);
      const float* dec_row = dec + row;
      bool ok = true;
      for (int c = 0; c < n_tiles; ++c) {
        const int t0 = (tile0 + c) * 128;
        const int m = min(128, sq.n_tokens - t0);
        const bool mixed = p.key_mask != nullptr || m < 128;
        uint32_t bits[2] = {~0u, ~0u};                        // of this thread's two column blocks
        if (mixed) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int j = 32 * (2 * b + half) + lane;
            bool valid = j < m;
            if (valid && p.key_mask != nullptr) valid = p.key_mask[sq.tok_start + t0 + j] != 0;
            bits[b] = __ballot_sync(0xffffffffu, valid);
          }
        }
        ok = __all_sync(0xffffffffu, mbar_wait(bar_s_full, c & 1, limit));
        if (!ok) break;
        tc_fence_after();
        // P of column block cb replaces the scores of that block, in its first 16 columns: a block is read and written by
        // one warp alone.  Blocks right of the diagonal are zero, left of it every decay exponent is positive.
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int cb = 2 * b + half;
          uint32_t pk[16];
          if (cb <= wq) {
            uint32_t s[32];
            tmem_ld32(tm + kColS + cb * 32, s);
            tmem_wait_ld();
            if (cb < wq && !mixed) {
              // g^{row - j} = g^{row - 32 cb - 31} * g^{31 - jj}: the second factor is the same for every row and tile
              const float lead = p.scale * dec_row[-cb * 32 - 31];
              const float2 lead2 = make_float2(lead, lead);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float4 d = fall[e];                      // g^{31 - 4 e}, ... - 1, - 2, - 3
                const float2 lo = mul_f32x2(make_float2(__uint_as_float(s[4 * e]), __uint_as_float(s[4 * e + 1])),
                                            mul_f32x2(lead2, make_float2(d.x, d.y)));
                const float2 hi = mul_f32x2(make_float2(__uint_as_float(s[4 * e + 2]), __uint_as_float(s[4 * e + 3])),
                                            mul_f32x2(lead2, make_float2(d.z, d.w)));
                pk[2 * e] = pack_bf16x2(lo.x, lo.y);
                pk[2 * e + 1] = pack_bf16x2(hi.x, hi.y);
              }
            } else {
              const float* d = dec_row - cb * 32;
              const int last = row - cb * 32;                  // columns beyond it lie above the diagonal
              const uint32_t on = bits[b] & (last >= 31 ? ~0u : (2u << last) - 1u);
#pragma unroll
              for (int e = 0; e < 16; ++e)
                pk[e] = pack_bf16x2((on >> (2 * e)) & 1u ? __uint_as_float(s[2 * e]) * (p.scale * d[-2 * e]) : 0.f,
                                    (on >> (2 * e + 1)) & 1u ? __uint_as_float(s[2 * e + 1]) * (p.scale * d[-2 * e - 1]) : 0.f);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) pk[e] = 0u;
          }
          tmem_st16(tm + kColS + cb * 32, pk);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p_full);

        ok = __all_sync(0xffffffffu, mbar_wait(bar_o_full, c & 1, limit));
        if (!ok) break;
        tc_fence_after();
        // The rows are staged where the tile's V was (nothing reads it any more), in the layout the TMA store expects.  A
        // tile that reaches beyond its sequence is written row by row instead: the rows behind it are not ours.
        const bool whole = m == 128;
        __nv_bfloat16* dst = p.out + (sq.tok_start + t0 + row) * p.o_tok_stride + (long long)head * p.o_head_stride + half * (D / 2);
        uint8_t* stage = smem + L::kOffV + (c % L::kStages) * L::kTile;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          const int cb = half * (D / 64) + i;
          uint32_t a[32], b[32];
          tmem_ld32(tm + kColO + cb * 32, a);
          tmem_ld32(tm + kColQS + cb * 32, b);
          tmem_wait_ld();
          if (i == D / 64 - 1) {                               // everything is in registers: the accumulators are free
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_o_empty);
          }
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const float2 x = fma_f32x2(g1_2, make_float2(__uint_as_float(b[8 * ch + e]), __uint_as_float(b[8 * ch + e + 1])),
                                         make_float2(__uint_as_float(a[8 * ch + e]), __uint_as_float(a[8 * ch + e + 1])));
              f[e] = x.x;
              f[e + 1] = x.y;
            }
            const int at = cb * 4 + ch;                        // 16-byte chunk of the row
            if (whole)         *reinterpret_cast<uint4*>(stage + (at >> 3) * 16384 + row * 128 + (((at & 7) ^ (row & 7)) << 4)) = pack8(f);
            else if (row < m)  *reinterpret_cast<uint4*>(dst + i * 32 + ch * 8) = pack8(f);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_o_staged);
      }
      if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutSoftmax);
    }
  } else if (warp < kTma) {
    // =========================================================== K -> K', state; two threads per token row / K dim
    if (!kStateOnly) setmaxnreg_inc<128>();
    const int wq = (warp - kFirstB) & 3, half = (warp - kFirstB) >> 2;
    const int row = wq * 32 + lane;
    constexpr int kCols = D / 2;                                           // columns of this thread's part of a row
    const uint32_t tm = tmem_base + (static_cast<uint32_t>(wq * 32) << 16) + kColT + half * kCols;
    float S[kCols];
#pragma unroll
    for (int e = 0; e < kCols; ++e) S[e] = 0.f;
    const bool has_state = row < D;                                        // warp-uniform
    // where this thread's 16-byte chunks of a row are in a tile (128-byte swizzle); D = 128: half = 64-column box
    auto chunk = [&](int ch, int box_bytes) {
      const int at = half * (kCols / 8) + ch;
      return (at >> 3) * box_bytes + row * 128 + (((at & 7) ^ (row & 7)) << 4);
    };
    auto publish = [&]() {
      // this part of the state's row, rounded to bf16, in the layout of a V tile (row = contraction index)
#pragma unroll
      for (int ch = 0; ch < kCols / 8; ++ch) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = S[ch * 8 + e];
        *reinterpret_cast<uint4*>(smem + L::kOffSt + chunk(ch, D * 128)) = pack8(f);
      }
      fence_proxy_async_smem();
    };
    // the state before this piece
    auto add_piece = [&](const float* piece, float g) {                    // S = g S + what a piece left in the workspace
      const float4* src = reinterpret_cast<const float4*>(piece) + half * (kCols / 4) * D + row;
#pragma unroll
      for (int e = 0; e < kCols / 4; ++e) {
        const float4 x = src[e * D];
        S[4 * e] = fmaf(g, S[4 * e], x.x); S[4 * e + 1] = fmaf(g, S[4 * e + 1], x.y);
        S[4 * e + 2] = fmaf(g, S[4 * e + 2], x.z); S[4 * e + 3] = fmaf(g, S[4 * e + 3], x.w);
      }
    };
    auto leave_piece = [&](float* piece) {
      float4* dst = reinterpret_cast<float4*>(piece) + half * (kCols / 4) * D + row;
#pragma unroll
      for (int e = 0; e < kCols / 4; ++e) dst[e * D] = make_float4(S[4 * e], S[4 * e + 1], S[4 * e + 2], S[4 * e + 3]);
    };
    if (has_state && seg == 0 && p.state_in != nullptr) {
      // A cut sequence: the state launch is the only one that reads state_in (its first piece starts from it and leaves a
      // copy), so that the main launch may write state_out to the same memory at any time.
      float* copy = p.initial + (long long)(si * p.heads + head) * (D * D);
      if (kStateOnly || n_seg == 1) {
        const float4* src = reinterpret_cast<const float4*>(p.state_in + (((long long)sq.seq_id * p.heads + head) * D + row) * D + half * kCols);
#pragma unroll
        for (int e = 0; e < kCols / 4; ++e) {
          const float4 x = src[e];
          S[4 * e] = x.x; S[4 * e + 1] = x.y; S[4 * e + 2] = x.z; S[4 * e + 3] = x.w;
        }
        if (kStateOnly) leave_piece(copy);
      } else {
        add_piece(copy, 0.f);
      }
    }
    if constexpr (!kStateOnly) {
      if (has_state) {
        const float gs = (float)exp(128.0 * p.seg_tiles * ld);             // every earlier segment is whole
        for (int r = 0; r < seg; ++r) add_piece(p.local + (long long)(local_first + r * p.heads + head) * (D * D), gs);
        publish();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_st_full);
    }
    // K' of this warp: K dims 32 wq .. + 31 (tensor-memory lanes), tokens 64 half .. + 63.  ldmatrix hands thread i the token
    // pairs 64 half + 8 t + 2 (i % 4), + 1 for t = 0..7: the weights of those 16 tokens, wb + wc, stay in registers.
    uint32_t wb[8], wc[8], on[8];                                          // on: all ones for a token that counts
    auto weights = [&](int m, const uint32_t (&bits)[2]) {
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        float w[2];
        on[t] = 0u;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int in = 8 * t + 2 * (lane & 3) + u, tok = 64 * half + in;
          const bool counts = ((bits[in >> 5] >> (in & 31)) & 1u) != 0;
          w[u] = counts ? dec[m - 1 - tok] : 0.f;
          if (counts) on[t] |= 0xffffu << (16 * u);
        }
        wb[t] = pack_bf16x2(w[0], w[1]);
        wc[t] = pack_bf16x2(w[0] - bf16_lo(wb[t]), w[1] - bf16_hi(wb[t]));
      }
    };
    {
      const uint32_t all[2] = {~0u, ~0u};
      weights(128, all);
    }
    // address of this lane's row in block (dim chunk dc, token block tb) of a K tile: lanes 0-7 and 16-23 the first 8 of 16
    // dims, the others the second 8; lanes 0-15 the first token block, the others the next
    const int tok_in = 64 * half + ((lane >> 4) << 3) + (lane & 7);
    const uint32_t k_row = tok_in * 128;
    const int dc_in = (lane >> 3) & 1;
    bool ok = true;
    int st = 0;
    uint32_t ph = 0;
    for (int c = 0; c < n_tiles; ++c) {
      const int t0 = (tile0 + c) * 128;
      const int m = min(128, sq.n_tokens - t0);
      const bool mixed = p.key_mask != nullptr || m < 128;
      uint32_t vbits = ~0u;                                                // of the 32 token rows 32 wq ..
      if (mixed) {
        uint32_t bits[2];
#pragma unroll
        for (int b = 0; b < 3; ++b) {
          const int j = (b < 2 ? 64 * half + 32 * b : 32 * wq) + lane;
          bool valid = j < m;
          if (valid && p.key_mask != nullptr) valid = p.key_mask[sq.tok_start + t0 + j] != 0;
          const uint32_t word = __ballot_sync(0xffffffffu, valid);
          if (b < 2) bits[b] = word; else vbits = word;
        }
        weights(m, bits);
      }
      ok = __all_sync(0xffffffffu, mbar_wait(bar_k_full(st), ph, limit));
      // the accumulators of the previous tile's outputs, whose columns K' takes, have been read
      if (!kStateOnly && c > 0) ok = ok && __all_sync(0xffffffffu, mbar_wait(bar_o_empty, (c - 1) & 1, limit));
      if (!ok) break;
      tc_fence_after();
      if (has_state) {
#pragma unroll
        for (int lh = 0; lh < 2; ++lh) {                                   // 16 of the 32 K dims
          const int dc = 4 * wq + 2 * lh + dc_in;                          // 16-byte chunk of the row
          const uint32_t src = sK + st * L::kTile + (dc >> 3) * 16384 + k_row + (((dc & 7) ^ (lane & 7)) << 4);
#pragma unroll
          for (int tg = 0; tg < 2; ++tg) {                                 // 32 tokens
            uint32_t x[2][4];
            ldmatrix_x4_trans(src + tg * 32 * 128, x[0]);
            ldmatrix_x4_trans(src + tg * 32 * 128 + 16 * 128, x[1]);
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
              const int t = tg * 4 + (r >> 1);                             // token block
              uint32_t k2 = x[r >> 2][r & 3];
              if (mixed) k2 &= on[t];                                      // whatever stands under a mask, NaN included, is dropped
              hi[r] = mul_bf16x2(k2, wb[t]);
              lo[r] = fma_bf16x2(k2, wc[t], fma_bf16x2(k2, wb[t], hi[r] ^ 0x80008000u));
            }
            const uint32_t dst = tmem_base + (static_cast<uint32_t>(wq * 32 + lh * 16) << 16) + kColO + half * 32 + tg * 16;
            tmem_st_16x128b_x4(dst, hi);
            tmem_st_16x128b_x4(dst + 64, lo);
          }
        }
        tmem_wait_st();
      }
      if (mixed) {
        // V rows that do not count become zeros: 0 * (whatever stands there) would not be 0 for infinities and NaN
        ok = __all_sync(0xffffffffu, mbar_wait(bar_v_full(st), ph, limit));
        if (!ok) break;
        if (((vbits >> lane) & 1u) == 0) {
#pragma unroll
          for (int ch = 0; ch < kCols / 8; ++ch)
            *reinterpret_cast<uint4*>(smem + L::kOffV + st * L::kTile + chunk(ch, 16384)) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_kp_full);

      ok = __all_sync(0xffffffffu, mbar_wait(bar_t_full, c & 1, limit));
      if (!ok) break;
      tc_fence_after();
      if (has_state) {
        const float gm = dec[m];
#pragma unroll
        for (int cb = 0; cb < kCols / 32; ++cb) {
          uint32_t t[32];
          tmem_ld32(tm + cb * 32, t);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 x = fma_f32x2(make_float2(gm, gm), make_float2(S[cb * 32 + e], S[cb * 32 + e + 1]),
                                       make_float2(__uint_as_float(t[e]), __uint_as_float(t[e + 1])));
            S[cb * 32 + e] = x.x;
            S[cb * 32 + e + 1] = x.y;
          }
        }
        tc_fence_before();
        if (!kStateOnly) publish();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_st_full);
      if (++st == L::kStages) { st = 0; ph ^= 1u; }
    }
    if (!ok) {
      if (lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutSoftmax);
    } else if (has_state) {
      if constexpr (kStateOnly) {
        leave_piece(p.local + (long long)(local_first + rel) * (D * D));
      } else if (seg == n_seg - 1 && p.state_out != nullptr) {
        float4* dst = reinterpret_cast<float4*>(p.state_out + (((long long)sq.seq_id * p.heads + head) * D + row) * D + half * kCols);
#pragma unroll
        for (int e = 0; e < kCols / 4; ++e) dst[e] = make_float4(S[4 * e], S[4 * e + 1], S[4 * e + 2], S[4 * e + 3]);
      }
    }
  } else if (!kStateOnly) {
    setmaxnreg_dec<48>();
  }
  if (warp == kTma) {
    // =========================================================== TMA producer
    if (lane == 0) {
      const uint64_t pol_once = l2_policy_evict_first();
      bool ok = true;
      int c = 0;
      for (; c < n_tiles && ok; ++c) {
        const int st = c % L::kStages, tok = tok0 + (tile0 + c) * 128;
        const uint32_t par = ((c / L::kStages) & 1) ^ 1u;
        if (!mbar_wait(bar_k_empty(st), par, limit)) { ok = false; break; }
        mbar_arrive_expect_tx(bar_k_full(st), L::kTile);
#pragma unroll
        for (int hf = 0; hf < L::kHalves; ++hf)
          tma_load_3d(sK + st * L::kTile + hf * 16384, &tm_k, bar_k_full(st), hf * 64, head, tok);
        if constexpr (!kStateOnly) {
          const int qs = c % L::kQStages;
          if (!mbar_wait(bar_q_empty(qs), ((c / L::kQStages) & 1) ^ 1u, limit)) { ok = false; break; }
          mbar_arrive_expect_tx(bar_q_full(qs), L::kTile);
#pragma unroll
          for (int hf = 0; hf < L::kHalves; ++hf)
            tma_load_3d_hint(sQ + qs * L::kTile + hf * 16384, &tm_q, bar_q_full(qs), hf * 64, head, tok, pol_once);
        }
        if (!mbar_wait(bar_v_empty(st), par, limit)) { ok = false; break; }
        mbar_arrive_expect_tx(bar_v_full(st), L::kTile);
#pragma unroll
        for (int hf = 0; hf < L::kHalves; ++hf)
          tma_load_3d(sV + st * L::kTile + hf * 16384, &tm_v, bar_v_full(st), hf * 64, head, tok);
      }
      if (!ok) {
        atomicCAS(p.status, 0u, kStatusTimeoutProducer);
        // copies still in flight land before the shared memory is given back: every stage's last phase that was begun
        for (int b = max(0, c - L::kStages); b <= c; ++b) {
          const int st = b % L::kStages;
          const uint32_t par = (b / L::kStages) & 1;
          if (b < c) { mbar_wait(bar_k_full(st), par, limit); mbar_wait(bar_v_full(st), par, limit); }
        }
        // the tile it gave up in: K (and Q) may have been asked for; a copy takes far less than the limit that has run out
      }
    }
    __syncwarp();
  } else if (warp == kMma) {
    // =========================================================== MMA issuer
    constexpr uint32_t idesc_qk = idesc_bf16_f32(128, 128, false);
    constexpr uint32_t idesc_d = idesc_bf16_f32(128, D, true);             // B MN-major: P V and Q S
    constexpr uint32_t kV_lbo = D == 128 ? 16384u : 16u, kSt_lbo = D == 128 ? 16384u : 16u;
    const uint32_t hi_desc = smem_desc_hi_sw128(1024);
    const uint32_t q_lo = smem_desc_lo(sQ, 16), k_lo = smem_desc_lo(sK, 16);
    const uint32_t v_lo = smem_desc_lo(sV, kV_lbo), st_lo = smem_desc_lo(sSt, kSt_lbo);
    constexpr uint32_t kStep = L::kTile >> 4;
    bool ok = true;
    int st = 0;
    uint32_t ph = 0;
    auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, limit); };
    for (int c = 0; c < n_tiles; ++c) {
      if (!wait(bar_k_full(st), ph)) { ok = false; break; }
      if constexpr (!kStateOnly) {
        const int qs = c % L::kQStages;
        if (!wait(bar_q_full(qs), (c / L::kQStages) & 1)) { ok = false; break; }
        tc_fence_after();
        // scores (the previous tile's P V, which read P there, was issued before)
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = ((k >> 2) * 16384 + (k & 3) * 32) >> 4;
          if (k == 0) mma_ss_elect<false>(tmem_base + kColS, q_lo + qs * kStep, k_lo + st * kStep, hi_desc, idesc_qk, 0u);
          else        mma_ss_elect<true>(tmem_base + kColS, q_lo + qs * kStep + off, k_lo + st * kStep + off, hi_desc, idesc_qk, 1u);
        }
        tc_commit_elect(bar_s_full);
        // Q times the state before this tile
        if (!wait(bar_st_full, c & 1)) { ok = false; break; }
        if (c > 0 && !wait(bar_o_empty, (c - 1) & 1)) { ok = false; break; }
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = ((k >> 2) * 16384 + (k & 3) * 32) >> 4;
          if (k == 0) mma_ss_elect<false>(tmem_base + kColQS, q_lo + qs * kStep, st_lo, hi_desc, idesc_d, 0u);
          else        mma_ss_elect<true>(tmem_base + kColQS, q_lo + qs * kStep + off, st_lo + k * (2048 >> 4), hi_desc, idesc_d, 1u);
        }
        tc_commit_elect(bar_q_empty(qs));
      } else {
        if (c > 0 && !wait(bar_st_full, (c - 1) & 1)) { ok = false; break; }         // K'^T V of the previous tile has been read
      }
      // what the tile adds to the state
      if (!wait(bar_v_full(st), ph)) { ok = false; break; }
      if (!wait(bar_kp_full, c & 1)) { ok = false; break; }
      tc_fence_after();
      // (D = 64: the upper 64 lanes hold no K dims; their rows of the product are never read)
#pragma unroll
      for (int k = 0; k < 16; ++k) {                                       // hi, then lo
        const uint32_t off = (k & 7) * (2048 >> 4);
        if (k == 0) mma_ts_elect<false>(tmem_base + kColT, tmem_base + kColO, v_lo + st * kStep, hi_desc, idesc_d, 0u);
        else        mma_ts_elect<true>(tmem_base + kColT, tmem_base + kColO + k * 8, v_lo + st * kStep + off, hi_desc, idesc_d, 1u);
      }
      tc_commit_elect(bar_t_full);
      tc_commit_elect(bar_k_empty(st));
      if constexpr (!kStateOnly) {
        if (!wait(bar_p_full, c & 1)) { ok = false; break; }
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t off = k * (2048 >> 4);
          if (k == 0) mma_ts_elect<false>(tmem_base + kColO, tmem_base + kColS, v_lo + st * kStep, hi_desc, idesc_d, 0u);
          else        mma_ts_elect<true>(tmem_base + kColO, tmem_base + kColS + (k >> 1) * 32 + (k & 1) * 8, v_lo + st * kStep + off, hi_desc, idesc_d, 1u);
        }
        tc_commit_elect(bar_o_full);
      } else {
        tc_commit_elect(bar_v_empty(st));                                  // (main launch: once the outputs staged there are on their way)
      }
      if (++st == L::kStages) { st = 0; ph ^= 1u; }
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
          const int st = c % L::kStages;
          if (!mbar_wait(bar_o_staged, c & 1, limit)) { atomicCAS(p.status, 0u, kStatusTimeoutSoftmax); break; }
          if (sq.n_tokens - (tile0 + c) * 128 >= 128) {
#pragma unroll
            for (int hf = 0; hf < L::kHalves; ++hf)
              tma_store_3d(&tm_o, sV + st * L::kTile + hf * 16384, hf * 64, head, tok0 + (tile0 + c) * 128);
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
