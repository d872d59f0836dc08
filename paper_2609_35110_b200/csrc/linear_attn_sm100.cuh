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
// is fp32 and carried from tile to tile, keeps about 17 bits of every factor instead of 8; the running state itself is
// never rounded below fp32 and never accumulated in tensor memory for longer than one tile.
//
// Warp roles:
//   warps 0-3   thread = query row: S-scores -> P, and the output epilogue
//   warps 4-7   thread = token row: K -> K' (hi in place of K, lo beside it); thread = K dim: row of the state
//   warp  8     TMA producer;   warp 9: MMA issuer, owns the tensor memory
// Tensor memory (512 columns): scores / P [0,128), P V [128,256), Q S [256,384), K'^T V [384,512).
// Bound by HBM: 4 x 128 x D x 2 bytes per tile and head against 5 (4 and the lo half) small products.
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

constexpr int kLinThreads = 320;

template <int D, bool kStateOnly>
struct LinearSmem {
  static constexpr int kTile = 128 * D * 2;
  static constexpr int kHalves = D / 64;
  static constexpr int kQStages = kStateOnly ? 0 : D == 128 ? 1 : 2;
  static constexpr int kStages = D == 128 ? 2 : 3;
  static constexpr int kOffQ = 0;
  static constexpr int kOffLo = kOffQ + kQStages * kTile;
  static constexpr int kOffK = kOffLo + kTile;
  static constexpr int kOffV = kOffK + kStages * kTile;
  static constexpr int kOffSt = kOffV + kStages * kTile;                 // bf16 copy of the state, laid out like V
  static constexpr int kOffDec = kOffSt + (kStateOnly ? 0 : D * D * 2);  // powers of the decay: [128 + d], zero for d < 0
  static constexpr int kOffBars = kOffDec + 264 * 4;
  static constexpr int kNumBars = 2 * kQStages + 4 * kStages + 8;
  static constexpr int kOffTmemPtr = kOffBars + kNumBars * 8;
  static constexpr int kBytes = kOffTmemPtr + 16;
  static constexpr int kDynBytes = kBytes + 1024;
};

// kind::f16 descriptor with both operands MN-major (bits 15 and 16)
__host__ __device__ constexpr uint32_t idesc_bf16_f32_tt(int M, int N) { return idesc_bf16_f32(M, N, true) | (1u << 15); }

__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ void st_shared_v4(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

template <int D, bool kStateOnly>
__global__ void __launch_bounds__(kLinThreads, 1)
linear_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const LinearParams p) {
  using L = LinearSmem<D, kStateOnly>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t sbase = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - raw_addr);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  const uint32_t sQ = sbase + L::kOffQ, sLo = sbase + L::kOffLo, sK = sbase + L::kOffK, sV = sbase + L::kOffV, sSt = sbase + L::kOffSt;
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
                 bar_o_empty = bars + 8u * (kSB + 6), bar_drain = bars + 8u * (kSB + 7);
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

  if (warp == 8 && lane == 0) {
    for (int s = 0; s < L::kQStages; ++s) { mbar_init(bar_q_full(s), 1); mbar_init(bar_q_empty(s), 1); }
    for (int s = 0; s < L::kStages; ++s) {
      mbar_init(bar_k_full(s), 1); mbar_init(bar_k_empty(s), 1);
      mbar_init(bar_v_full(s), 1); mbar_init(bar_v_empty(s), 1);
    }
    mbar_init(bar_s_full, 1);
    mbar_init(bar_p_full, 4);
    mbar_init(bar_kp_full, 4);
    mbar_init(bar_t_full, 1);
    mbar_init(bar_st_full, 4);
    mbar_init(bar_o_full, 1);
    mbar_init(bar_o_empty, 4);
    mbar_init(bar_drain, 1);
    fence_mbar_init();
    if (!kStateOnly) prefetch_tensormap(&tm_q);
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  if (threadIdx.x == 0) tmem_ptr_smem[1] = *reinterpret_cast<volatile unsigned int*>(p.status);
  if (warp == 9) { tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_ptr_smem)), 512); tmem_relinquish(); }
  const double ld = fmin((double)__ldg(p.log_decay + head), 0.0);
  if (threadIdx.x < 257) {
    const int d = (int)threadIdx.x - 128;
    dec[d] = d < 0 ? 0.f : d == 0 ? 1.f : (float)exp((double)d * ld);     // (0 * -inf is NaN: g^0 is 1)
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_ptr_smem[0];
  if (tmem_ptr_smem[1] != 0) {                             // a fault recorded earlier stops later CTAs at the door
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem_base, 512);
    return;
  }
  constexpr uint32_t kColS = 0, kColO = 128, kColQS = 256, kColT = 384;

  if (warp < 4) {
    if constexpr (!kStateOnly) {
      // =========================================================== scores -> P, outputs; thread = query row
      const int row = warp * 32 + lane;
      const uint32_t tm = tmem_base + (static_cast<uint32_t>(warp * 32) << 16);
      const float g1 = dec[row + 1];
      bool ok = true;
      for (int c = 0; c < n_tiles; ++c) {
        const int t0 = (tile0 + c) * 128;
        const int m = min(128, sq.n_tokens - t0);
        uint32_t bits[4] = {~0u, ~0u, ~0u, ~0u};
        if (p.key_mask != nullptr || m < 128) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            bool valid = 32 * w + lane < m;
            if (valid && p.key_mask != nullptr) valid = p.key_mask[sq.tok_start + t0 + 32 * w + lane] != 0;
            bits[w] = __ballot_sync(0xffffffffu, valid);
          }
        }
        ok = __all_sync(0xffffffffu, mbar_wait(bar_s_full, c & 1, limit));
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          uint32_t pk[16];
          if (cb <= warp) {
            uint32_t s[32];
            tmem_ld32(tm + kColS + cb * 32, s);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float f[2];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const int j = cb * 32 + 2 * e + u;
                const bool on = j <= row && ((bits[cb] >> (2 * e + u)) & 1u) != 0;
                f[u] = on ? __uint_as_float(s[2 * e + u]) * dec[row - j] : 0.f;
              }
              pk[e] = pack_bf16x2(f[0], f[1]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) pk[e] = 0u;                       // above the diagonal
          }
          // columns [16 cb, 16 cb + 16) hold scores of blocks <= cb / 2, which are in registers or done with
          tmem_st16(tm + kColS + cb * 16, pk);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p_full);

        ok = __all_sync(0xffffffffu, mbar_wait(bar_o_full, c & 1, limit));
        if (!ok) break;
        tc_fence_after();
        const bool store = row < m;
        // even lanes store 32 bytes of their own row, then of their neighbour's, and so do odd ones: whole sectors
        const int peer_row = t0 + (row ^ 1);
        __nv_bfloat16* mine = p.out + (sq.tok_start + t0 + row) * p.o_tok_stride + (long long)head * p.o_head_stride;
        __nv_bfloat16* theirs = p.out + (sq.tok_start + peer_row) * p.o_tok_stride + (long long)head * p.o_head_stride;
        const bool store_peer = (row ^ 1) < m;
        const bool odd = lane & 1;
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) {
          uint32_t a[32], b[32];
          tmem_ld32(tm + kColO + cb * 32, a);
          tmem_ld32(tm + kColQS + cb * 32, b);
          tmem_wait_ld();
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e)
            w[e] = pack_bf16x2(p.scale * fmaf(g1, __uint_as_float(b[2 * e]), __uint_as_float(a[2 * e])),
                               p.scale * fmaf(g1, __uint_as_float(b[2 * e + 1]), __uint_as_float(a[2 * e + 1])));
#pragma unroll
          for (int h = 0; h < 2; ++h) {                                    // 16 values = two 16-byte chunks
            uint32_t own[4], give[4], got[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              own[e] = odd ? w[8 * h + 4 + e] : w[8 * h + e];              // even lanes keep chunk 0, odd ones chunk 1
              give[e] = odd ? w[8 * h + e] : w[8 * h + 4 + e];
              got[e] = __shfl_xor_sync(0xffffffffu, give[e], 1);
            }
            const int col = cb * 32 + h * 16 + (odd ? 8 : 0);
            // first the even row's two chunks, then the odd row's
            const uint4 first_w = odd ? make_uint4(got[0], got[1], got[2], got[3]) : make_uint4(own[0], own[1], own[2], own[3]);
            const uint4 second_w = odd ? make_uint4(own[0], own[1], own[2], own[3]) : make_uint4(got[0], got[1], got[2], got[3]);
            if (odd ? store_peer : store) *reinterpret_cast<uint4*>((odd ? theirs : mine) + col) = first_w;
            if (odd ? store : store_peer) *reinterpret_cast<uint4*>((odd ? mine : theirs) + col) = second_w;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_o_empty);
      }
      if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutSoftmax);
    }
  } else if (warp < 8) {
    // =========================================================== K -> K', state; thread = token row, then K dim
    const int row = (warp - 4) * 32 + lane;
    const uint32_t tm = tmem_base + (static_cast<uint32_t>((warp - 4) * 32) << 16);
    float S[D];
#pragma unroll
    for (int e = 0; e < D; ++e) S[e] = 0.f;
    const bool has_state = row < D;                                        // warp-uniform
    auto publish = [&]() {
      // row of the state, rounded to bf16, in the layout of a V tile (row = contraction index)
#pragma unroll
      for (int ch = 0; ch < D / 8; ++ch) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = S[ch * 8 + e];
        st_shared_v4(sSt + (ch >> 3) * (D * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4), pack8(f));
      }
      fence_proxy_async_smem();
    };
    // the state before this piece
    auto add_piece = [&](const float* piece, float g) {                    // S = g S + what a piece left in the workspace
      const float4* src = reinterpret_cast<const float4*>(piece) + row;
#pragma unroll
      for (int e = 0; e < D / 4; ++e) {
        const float4 x = src[e * D];
        S[4 * e] = fmaf(g, S[4 * e], x.x); S[4 * e + 1] = fmaf(g, S[4 * e + 1], x.y);
        S[4 * e + 2] = fmaf(g, S[4 * e + 2], x.z); S[4 * e + 3] = fmaf(g, S[4 * e + 3], x.w);
      }
    };
    auto leave_piece = [&](float* piece) {
      float4* dst = reinterpret_cast<float4*>(piece) + row;
#pragma unroll
      for (int e = 0; e < D / 4; ++e) dst[e * D] = make_float4(S[4 * e], S[4 * e + 1], S[4 * e + 2], S[4 * e + 3]);
    };
    if (has_state && seg == 0 && p.state_in != nullptr) {
      // A cut sequence: the state launch is the only one that reads state_in (its first piece starts from it and leaves a
      // copy), so that the main launch may write state_out to the same memory at any time.
      float* copy = p.initial + (long long)(si * p.heads + head) * (D * D);
      if (kStateOnly || n_seg == 1) {
        const float4* src = reinterpret_cast<const float4*>(p.state_in + (((long long)sq.seq_id * p.heads + head) * D + row) * D);
#pragma unroll
        for (int e = 0; e < D / 4; ++e) {
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
    bool ok = true;
    int st = 0;
    uint32_t ph = 0;
    for (int c = 0; c < n_tiles; ++c) {
      const int t0 = (tile0 + c) * 128;
      const int m = min(128, sq.n_tokens - t0);
      bool valid = row < m;
      if (valid && p.key_mask != nullptr) valid = p.key_mask[sq.tok_start + t0 + row] != 0;
      const float w = valid ? dec[m - 1 - row] : 0.f;
      ok = __all_sync(0xffffffffu, mbar_wait(bar_k_full(st), ph, limit));
      if (!kStateOnly) ok = ok && __all_sync(0xffffffffu, mbar_wait(bar_s_full, c & 1, limit));   // K has been multiplied with Q
      if (!ok) break;
#pragma unroll
      for (int ch = 0; ch < D / 8; ++ch) {
        const uint32_t off = (ch >> 3) * 16384 + row * 128 + (((ch & 7) ^ (row & 7)) << 4);
        uint4 hi = make_uint4(0, 0, 0, 0), lo = make_uint4(0, 0, 0, 0);
        if (valid) {
          float f[8], r[8];
          unpack8(ld_shared_v4(sK + st * L::kTile + off), f);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] *= w;
          hi = pack8(f);
          unpack8(hi, r);
#pragma unroll
          for (int e = 0; e < 8; ++e) r[e] = f[e] - r[e];
          lo = pack8(r);
        }
        st_shared_v4(sK + st * L::kTile + off, hi);
        st_shared_v4(sLo + off, lo);
      }
      if (m < 128 || p.key_mask != nullptr) {
        // V rows that do not count become zeros: 0 * (whatever stands there) would not be 0 for infinities and NaN
        ok = __all_sync(0xffffffffu, mbar_wait(bar_v_full(st), ph, limit));
        if (!ok) break;
        if (!valid) {
#pragma unroll
          for (int ch = 0; ch < D / 8; ++ch)
            st_shared_v4(sV + st * L::kTile + (ch >> 3) * 16384 + row * 128 + ((ch & 7) << 4), make_uint4(0, 0, 0, 0));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_kp_full);

      ok = __all_sync(0xffffffffu, mbar_wait(bar_t_full, c & 1, limit));
      if (!ok) break;
      tc_fence_after();
      if (has_state) {
        const float gm = dec[m];
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) {
          uint32_t t[32];
          tmem_ld32(tm + kColT + cb * 32, t);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) S[cb * 32 + e] = fmaf(gm, S[cb * 32 + e], __uint_as_float(t[e]));
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
        float4* dst = reinterpret_cast<float4*>(p.state_out + (((long long)sq.seq_id * p.heads + head) * D + row) * D);
#pragma unroll
        for (int e = 0; e < D / 4; ++e) dst[e] = make_float4(S[4 * e], S[4 * e + 1], S[4 * e + 2], S[4 * e + 3]);
      }
    }
  } else if (warp == 8) {
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
  } else {
    // =========================================================== MMA issuer
    constexpr uint32_t idesc_qk = idesc_bf16_f32(128, 128, false);
    constexpr uint32_t idesc_d = idesc_bf16_f32(128, D, true);             // B MN-major: P V and Q S
    constexpr uint32_t idesc_t = idesc_bf16_f32_tt(128, D);                // A and B MN-major: K'^T V
    constexpr uint32_t kV_lbo = D == 128 ? 16384u : 16u, kSt_lbo = D == 128 ? 16384u : 16u;
    const uint32_t hi_desc = smem_desc_hi_sw128(1024);
    const uint32_t q_lo = smem_desc_lo(sQ, 16), k_lo = smem_desc_lo(sK, 16);
    const uint32_t v_lo = smem_desc_lo(sV, kV_lbo), st_lo = smem_desc_lo(sSt, kSt_lbo);
    // K' as the A operand, M = 128 K dims.  With D = 64 the upper 64 rows come from whatever lies 16 KB further on (inside
    // this CTA's shared memory) and end in tensor-memory lanes that nobody reads.
    const uint32_t kt_lo = smem_desc_lo(sK, 16384), lo_lo = smem_desc_lo(sLo, 16384);
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
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t off = k * (2048 >> 4);
        if (k == 0) mma_ss_elect<false>(tmem_base + kColT, kt_lo + st * kStep, v_lo + st * kStep, hi_desc, idesc_t, 0u);
        else        mma_ss_elect<true>(tmem_base + kColT, kt_lo + st * kStep + off, v_lo + st * kStep + off, hi_desc, idesc_t, 1u);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t off = k * (2048 >> 4);
        mma_ss_elect<true>(tmem_base + kColT, lo_lo + off, v_lo + st * kStep + off, hi_desc, idesc_t, 1u);
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
          else        mma_ts_elect<true>(tmem_base + kColO, tmem_base + kColS + k * 8, v_lo + st * kStep + off, hi_desc, idesc_d, 1u);
        }
        tc_commit_elect(bar_o_full);
      }
      tc_commit_elect(bar_v_empty(st));
      if (++st == L::kStages) { st = 0; ph ^= 1u; }
    }
    if (!ok) {
      if (lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutMma);
      tc_commit_elect(bar_drain);
      mbar_wait_warp(bar_drain, 0, limit);
    }
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

}  // namespace sol
