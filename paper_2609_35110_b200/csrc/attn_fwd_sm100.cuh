// Attention main kernel for sm_100a: S = Q~ K~^T and O += P V on tcgen05 tensor cores with the
// accumulators in tensor memory, TMA-fed shared-memory ring, online softmax in registers.
//
// One CTA = one (sequence, head, pair of 128-row query tiles).  With kCtas = 2 two such CTAs on neighbouring SMs
// form a cluster that covers 512 consecutive query rows of one (sequence, head) and shares every K / V tile:
// each CTA loads HALF of the tile (K: 64 of the 128 keys; V: 64 of the 128 head dims) with its own TMA loads and
// one tcgen05.mma.cta_group::2 of M = 256 works on both CTAs' query rows, which halves the shared-memory reads of
// the B operand and the L2 -> SM traffic per flop.  The even CTA (the leader) issues all MMAs; completion goes to
// both CTAs with a multicast commit.  Nothing is loaded with multicast.
// Warp roles (per CTA):
//   warps 0-3   softmax / correction / epilogue of query tile 0 (thread = one query row)
//   warps 4-7   the same for query tile 1
//   warp  8     TMA producer (lane 0)
//   warp  9     tcgen05.mma issuer: the whole warp runs the loop convergently, one elected lane issues each
//               instruction (descriptors then stay in uniform registers); owns the TMEM allocation
//   warps 10-11 idle (complete the third warpgroup)
// (differential attention: 0-15 softmax, 16 producer, 17 and 18 issuers, 19 looks up V's exponent, 20-23 convert V; see kDiff below)
// The two query tiles ping-pong: while the softmax of one tile runs on the ALUs, the tensor core
// works on the other tile's QK^T / PV.
//
// Tensor memory (512 columns x 128 lanes x 32 bit):
//   [0,128)    S0  (fp32 scores of tile 0);  P0 (bf16, 64 columns) overwrites its first half
//   [128,256)  S1 / P1
//   [256,256+D)       O0 (fp32)
//   [256+D,256+2D)    O1
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "device_types.cuh"
#include "exchange_kernels.cuh"
#include "ptx_sm100.cuh"

namespace sol {

// Register split after launch (384 threads x 168): the softmax warpgroups take what the third
// warpgroup (producer, MMA issuer, two idle warps) gives back: (168 - other) * 128 >= (softmax - 168) * 256.
#ifndef SOL_REGS_SOFTMAX
#define SOL_REGS_SOFTMAX 216
#endif
#ifndef SOL_REGS_OTHER
#define SOL_REGS_OTHER 64
#endif
constexpr int kDiffThreads = 768;   // 16 softmax warps, producer, an MMA issuer per map, a warp with little to do, 4 warps that convert V
constexpr int kAttnThreads = 384;   // 8 softmax warps + producer + MMA issuer + 2 idle warps (a full third warpgroup)

__device__ __forceinline__ float row_max128(const uint32_t (&r)[128]) {
  float m0 = max3(__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[2]));
  float m1 = max3(__uint_as_float(r[3]), __uint_as_float(r[4]), __uint_as_float(r[5]));
#pragma unroll
  for (int cc = 6; cc + 3 < 128; cc += 4) {
    m0 = max3(m0, __uint_as_float(r[cc]), __uint_as_float(r[cc + 1]));
    m1 = max3(m1, __uint_as_float(r[cc + 2]), __uint_as_float(r[cc + 3]));
  }
  return max3(m0, m1, fmaxf(__uint_as_float(r[126]), __uint_as_float(r[127])));
}

// One pass over a 128-column score row held in registers: p = 2^(s*c - mc) packed to bf16 and the fp32
// row sum of the un-rounded p.  Every exponential goes to the special-function unit: evaluating a share of them
// with a polynomial on the FMA pipes was measured more than once (scalar and packed fp32x2 arithmetic, 1/8 to 1/2
// of the elements) and lost every time: the polynomial costs 12 to 16 issue cycles per element against 8
// special-function cycles, and the thread-per-row layout has no registers left to interleave enough of them.
__device__ __forceinline__ void softmax_pass(const uint32_t (&r)[128], float c, float mc, uint32_t (&pk)[64],
                                             float& sum) {
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int cc = 0; cc < 64; ++cc) {
    const float p_lo = ex2_approx(fmaf(__uint_as_float(r[2 * cc]), c, -mc));
    const float p_hi = ex2_approx(fmaf(__uint_as_float(r[2 * cc + 1]), c, -mc));
    acc[(2 * cc) & 3] += p_lo;
    acc[(2 * cc + 1) & 3] += p_hi;
    pk[cc] = pack_bf16x2(p_lo, p_hi);
  }
  sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

// Address of output row (flat token, head) in the destination that owns the token.
__device__ __forceinline__ uint8_t* out_row_ptr(const AttnParams& p, long long tok, int head, int elem_bytes) {
  int g = 0;
  while (g + 1 < p.sink.n_dst && tok >= p.sink.tok_begin[g + 1]) ++g;
  return static_cast<uint8_t*>(p.sink.base[g]) +
         ((tok - p.sink.tok_begin[g]) * p.o_tok_stride + (long long)head * p.o_head_stride) * elem_bytes;
}

// Writes a warp's 32 staged rows (16-byte chunks XOR-swizzled by row) to global memory, one chunk per lane.
// byte0: the chunks' offset in the output row.
template <int kRowBytes>
__device__ __forceinline__ void write_staged_rows(const AttnParams& p, const SeqDev& sq, int head, int first_row, int lane,
                                                  int elem_bytes, const uint8_t* stage, int byte0 = 0) {
  constexpr int kLanesPerRow = kRowBytes / 16;
  __syncwarp();
  const uint64_t pol_once = l2_policy_evict_first();            // output rows are written once, never read here
  const int ch = lane % kLanesPerRow;
#pragma unroll 4
  for (int r0 = 0; r0 < 32; r0 += 32 / kLanesPerRow) {
    const int rr = r0 + lane / kLanesPerRow;
    const int qrow = first_row + rr;
    bool store = qrow < sq.n_tokens;
    if (store && p.query_mask != nullptr) store = p.query_mask[sq.tok_start + qrow] != 0;
    SOL_DEVICE_CHECK(p.status, !store || (sq.tok_start + qrow >= 0 && sq.tok_start + qrow < p.sink.tok_begin[p.sink.n_dst]),
                     kCheckOutputRow);
    const uint4 w = *reinterpret_cast<const uint4*>(stage + rr * kRowBytes + ((ch ^ (rr & (kLanesPerRow - 1))) << 4));
    if (store) st_global_evict_first(out_row_ptr(p, sq.tok_start + qrow, head, elem_bytes) + byte0 + ch * 16, w, pol_once);
  }
}

// Epilogue of one warp: its 32 accumulator rows O * inv -> bf16 (or raw E4M3 bytes) -> staged in the part of
// the query tile's shared memory that belongs to those rows (every MMA that read it has completed; 16-byte
// chunks XOR-swizzled by row) -> written out with one 16-byte chunk per lane, so every store instruction
// covers whole contiguous rows.  Rows beyond the sequence, or not wanted by the query mask, are not stored.
template <int D, bool kFp8>
__device__ __forceinline__ void store_rows(const AttnParams& p, const SeqDev& sq, int head, int first_row, int lane,
                                           uint32_t tO, float inv, uint8_t* stage) {
  constexpr int kRowBytes = kFp8 ? D : D * 2;
  constexpr int kLanesPerRow = kRowBytes / 16;
#pragma unroll
  for (int cch = 0; cch < D / 32; ++cch) {
    uint32_t o[32];
    tmem_ld32(tO + cch * 32, o);
    tmem_wait_ld();
    if (kFp8) {
#pragma unroll
      for (int v4 = 0; v4 < 2; ++v4) {
        uint4 w;
        w.x = pack_e4m3x4(__uint_as_float(o[16 * v4 + 0]) * inv, __uint_as_float(o[16 * v4 + 1]) * inv,
                          __uint_as_float(o[16 * v4 + 2]) * inv, __uint_as_float(o[16 * v4 + 3]) * inv);
        w.y = pack_e4m3x4(__uint_as_float(o[16 * v4 + 4]) * inv, __uint_as_float(o[16 * v4 + 5]) * inv,
                          __uint_as_float(o[16 * v4 + 6]) * inv, __uint_as_float(o[16 * v4 + 7]) * inv);
        w.z = pack_e4m3x4(__uint_as_float(o[16 * v4 + 8]) * inv, __uint_as_float(o[16 * v4 + 9]) * inv,
                          __uint_as_float(o[16 * v4 + 10]) * inv, __uint_as_float(o[16 * v4 + 11]) * inv);
        w.w = pack_e4m3x4(__uint_as_float(o[16 * v4 + 12]) * inv, __uint_as_float(o[16 * v4 + 13]) * inv,
                          __uint_as_float(o[16 * v4 + 14]) * inv, __uint_as_float(o[16 * v4 + 15]) * inv);
        const int ch = cch * 2 + v4;
        *reinterpret_cast<uint4*>(stage + lane * kRowBytes + ((ch ^ (lane & (kLanesPerRow - 1))) << 4)) = w;
      }
    } else {
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        uint4 w;
        w.x = pack_bf16x2(__uint_as_float(o[8 * v4 + 0]) * inv, __uint_as_float(o[8 * v4 + 1]) * inv);
        w.y = pack_bf16x2(__uint_as_float(o[8 * v4 + 2]) * inv, __uint_as_float(o[8 * v4 + 3]) * inv);
        w.z = pack_bf16x2(__uint_as_float(o[8 * v4 + 4]) * inv, __uint_as_float(o[8 * v4 + 5]) * inv);
        w.w = pack_bf16x2(__uint_as_float(o[8 * v4 + 6]) * inv, __uint_as_float(o[8 * v4 + 7]) * inv);
        const int ch = cch * 4 + v4;
        *reinterpret_cast<uint4*>(stage + lane * kRowBytes + ((ch ^ (lane & (kLanesPerRow - 1))) << 4)) = w;
      }
    }
  }
  write_staged_rows<kRowBytes>(p, sq, head, first_row, lane, kFp8 ? 1 : 2, stage);
}

// Epilogue in the block-INT8 wire format of the exchange (Section 3.2, "Quantized communication"): the thread that owns
// an accumulator row writes that row's record, [D int8 | D/32 scale codes | zeros to a multiple of 16 bytes], straight
// from tensor memory.  A group of 32 values is exactly one 32-column load.  The values are first rounded to bf16 and
// then quantised by the rule of quantize_records_kernel, so the bytes equal those of the bf16 epilogue followed by that
// kernel; what is saved is a write and a read of the bf16 rows.  A record is contiguous (144 bytes at D = 128), so
// every thread writes whole 16-byte chunks of its own record; nothing is staged.
template <int D>
__device__ __forceinline__ void store_rows_int8(const AttnParams& p, const SeqDev& sq, int head, int qrow, uint32_t tO, float inv) {
  constexpr int kGroups = D / 32;
  constexpr int kRecBytes = (D + kGroups + 15) / 16 * 16;
  bool store = qrow < sq.n_tokens;
  if (store && p.query_mask != nullptr) store = p.query_mask[sq.tok_start + qrow] != 0;
  SOL_DEVICE_CHECK(p.status, !store || sq.tok_start + qrow < p.sink.tok_begin[p.sink.n_dst], kCheckOutputRow);
  uint8_t* rec = out_row_ptr(p, sq.tok_start + (store ? qrow : 0), head, 1);
  uint32_t codes = 0;
#pragma unroll
  for (int grp = 0; grp < kGroups; ++grp) {
    uint32_t o[32];
    tmem_ld32(tO + grp * 32, o);                  // warp-collective: every lane loads, whether or not its row is stored
    tmem_wait_ld();
    float f[32];
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      f[e] = __bfloat162float(__float2bfloat16_rn(__uint_as_float(o[e]) * inv));
      amax = fmaxf(amax, fabsf(f[e]));
    }
    const int code = ue5m3_smallest_cover(amax);
    const float rs = __frcp_rn(ue5m3_value(code));
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      w[j] = pack_low_bytes(rint_sat_s8(__fmul_rn(f[4 * j], rs)), rint_sat_s8(__fmul_rn(f[4 * j + 1], rs)),
                            rint_sat_s8(__fmul_rn(f[4 * j + 2], rs)), rint_sat_s8(__fmul_rn(f[4 * j + 3], rs)));
    codes |= (uint32_t)code << (8 * grp);
    if (store) {
      uint4* dst = reinterpret_cast<uint4*>(rec + grp * 32);
      dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
      dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
  // tail: the scale codes, then zeros up to the record size (D = 128: one chunk; D = 64: 2 codes + 14 zeros)
  if (store) {
#pragma unroll
    for (int b = D; b < kRecBytes; b += 16)
      *reinterpret_cast<uint4*>(rec + b) = make_uint4(b == D ? codes : 0u, 0u, 0u, 0u);
  }
}

// Half of softmax_pass: 64 columns -> 32 packed pairs, partial sums kept in acc.
__device__ __forceinline__ void softmax_half(const uint32_t (&r)[64], float c, float mc, uint32_t (&pk)[32], float (&acc)[4]) {
#pragma unroll
  for (int cc = 0; cc < 32; ++cc) {
    const float p_lo = ex2_approx(fmaf(__uint_as_float(r[2 * cc]), c, -mc));
    const float p_hi = ex2_approx(fmaf(__uint_as_float(r[2 * cc + 1]), c, -mc));
    acc[(2 * cc) & 3] += p_lo;
    acc[(2 * cc + 1) & 3] += p_hi;
    pk[cc] = pack_bf16x2(p_lo, p_hi);
  }
}

template <int D, int kCtas = 1, bool kDiff = false>
struct AttnSmem {
  static constexpr int kTile = 128 * D * 2;               // bytes of one 128 x D bf16 tile
  static constexpr int kHalves = D / 64;                  // 64-column (128-byte) swizzle boxes per row
  static constexpr int kHalfBytes = 128 * 128;            // one box: 128 rows x 128 bytes
  static constexpr int kStageBytes = kTile / kCtas;       // what one CTA holds of a K or V tile
  static constexpr int kKBoxBytes = kHalfBytes / kCtas;   // one K box: (128 / kCtas) keys x 128 bytes
  // K/V ring (K and V tiles alternate); differential attention has one Q tile instead of two: its bytes go to the ring
  static constexpr int kStages = kDiff ? 10 : ((D == 128) ? 5 : 10) * (kCtas == 2 ? 8 : 5) / 5;
  static constexpr int kOffQ = 0;
  static constexpr int kOffKV = (kDiff ? 1 : 2) * kTile;
  static constexpr int kOffBars = kOffKV + kStages * kStageBytes;
  // q_full, kv_full/empty, s_full[2], p_full[2], o_done[2], drain; differential attention: v_ready per stage, s_full, p_full and
  // o_done of the second buffers, a second drain
  static constexpr int kNumBars = 1 + 2 * kStages + 7 + (kDiff ? kStages + 7 : 0);
  static constexpr int kOffTmemPtr = kOffBars + kNumBars * 8;
  static constexpr int kOffXchg = kOffTmemPtr + 16;       // differential attention: row sums [2][128], sums of squares [4][128], fp32
  static constexpr int kBytes = kOffXchg + (kDiff ? 6 * 128 * 4 : 0);
  static constexpr int kDynBytes = kBytes + 1024;         // slack to align the base to 1024 bytes
};

// The parts of the differential epilogue exchange through shared memory: a barrier over the sixteen softmax warps.
__device__ __forceinline__ void softmax_warps_sync() { asm volatile("bar.sync 1, 512;" ::: "memory"); }

// lambda of one head pair, by one warp (every lane gets it).
__device__ __forceinline__ float diff_lambda(const DiffWeightsDev& w, int pair, int lane) {
  float dot[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const float* a = w.vec[2 * m] + (long long)pair * w.pair_stride;
    const float* b = w.vec[2 * m + 1] + (long long)pair * w.pair_stride;
    dot[m] = __ldg(a + lane) * __ldg(b + lane) + __ldg(a + 32 + lane) * __ldg(b + 32 + lane);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot[m] += __shfl_xor_sync(0xffffffffu, dot[m], o);
  }
  return expf(dot[0]) - expf(dot[1]) + w.lambda_init;
}

// 128 validity bits of a key tile when no mask is given: the tokens the sequence has.
__device__ __forceinline__ uint4 tail_bits(int rem) {
  auto word = [](int r) { return r >= 32 ? 0xffffffffu : r <= 0 ? 0u : (1u << r) - 1u; };
  return make_uint4(word(rem), word(rem - 32), word(rem - 64), word(rem - 96));
}

// Epilogue of the differential attention.  Query tile t of the kernel is softmax map t over the same 128 rows, so a row of
// map 0 and the same row of map 1 are in the same tensor-memory lane.  Thread = row: the warps (t, h) combine columns
// [64 t + 32 h, + 32) of both accumulators, O0 / l0 - lambda * O1 / l1, which is a half of head 2 * pair + t of the output.  The
// norm's sums of squares cross over through shared memory and are added in a fixed order.
template <typename L>
__device__ __forceinline__ void diff_epilogue(const AttnParams& p, const SeqDev& sq, int pair, int t, int h, int first_row, int lane,
                                              int wq, uint32_t tmem_lane, float lam, uint8_t* smem) {
  const int v_exp = reinterpret_cast<const int*>(smem + L::kOffTmemPtr)[2];
  const float* xl = reinterpret_cast<const float*>(smem + L::kOffXchg);    // [map][row] row sums
  float* xs = reinterpret_cast<float*>(smem + L::kOffXchg) + 256;          // [map][half][row] sums of squares
  const int row = wq * 32 + lane;
  const float a0 = 1.0f / xl[row], a1 = lam / xl[128 + row];
  float x[32];
  float ss = 0.f;
#pragma unroll
  for (int e0 = 0; e0 < 32; e0 += 16) {
    uint32_t o0[16], o1[16];
    tmem_ld16(tmem_lane + 256 + t * 64 + h * 32 + e0, o0);
    tmem_ld16(tmem_lane + 384 + t * 64 + h * 32 + e0, o1);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      x[e0 + e] = __uint_as_float(o0[e]) * a0 - __uint_as_float(o1[e]) * a1;
      ss = fmaf(x[e0 + e], x[e0 + e], ss);
    }
  }
  if (p.diff.gain != nullptr) {
    xs[(2 * t + h) * 128 + row] = ss;
    softmax_warps_sync();
    ss = (xs[row] + xs[128 + row]) + (xs[256 + row] + xs[384 + row]);
    // x is held times 2^-v_exp; eps joins it in that scale.  If that leaves fp32's range upwards, eps is all that counts; if
    // downwards, it still keeps a row of zeros from 0 / 0.
    const float up = power_of_two(-v_exp), eps = p.diff.eps * up * up;
    float norm = eps < CUDART_INF_F ? sqrtf(fmaf(ss, 1.0f / 128.0f, eps)) : sqrtf(p.diff.eps) * up;
    if (norm == 0.f && p.diff.eps > 0.f) norm = 1.f;
    const float f = (1.0f - p.diff.lambda_init) / norm;
    const float4* g4 = reinterpret_cast<const float4*>(p.diff.gain + t * 64 + h * 32);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float4 g = __ldg(g4 + e);
      x[4 * e] *= f * g.x; x[4 * e + 1] *= f * g.y; x[4 * e + 2] *= f * g.z; x[4 * e + 3] *= f * g.w;
    }
  } else {
    const float f = power_of_two(v_exp);
#pragma unroll
    for (int e = 0; e < 32; ++e) x[e] *= f;
  }
  // every MMA has completed: the Q tile is the staging buffer, 2 KB per warp
  uint8_t* stage = smem + L::kOffQ + ((2 * t + h) * 4 + wq) * 32 * 64;
#pragma unroll
  for (int ch = 0; ch < 4; ++ch) {
    uint4 w;
    w.x = pack_bf16x2(x[8 * ch], x[8 * ch + 1]);
    w.y = pack_bf16x2(x[8 * ch + 2], x[8 * ch + 3]);
    w.z = pack_bf16x2(x[8 * ch + 4], x[8 * ch + 5]);
    w.w = pack_bf16x2(x[8 * ch + 6], x[8 * ch + 7]);
    *reinterpret_cast<uint4*>(stage + lane * 64 + ((ch ^ (lane & 3)) << 4)) = w;
  }
  write_staged_rows<64>(p, sq, 2 * pair + t, first_row, lane, 2, stage, h * 64);
}

// Softmax of the differential attention: warps 8 t .. 8 t + 7 serve map t, 64 keys per step (keys 32 b .. + 31 and 64 + 32 b
// .. + 31 of a tile: a CTA pair splits the tile's keys in two).  A map has two score buffers of 64 columns, so that the tensor
// core computes the next step's scores while this one is exponentiated.  A warp has 16 rows, in the layout of a matrix
// fragment: thread i holds columns 8 n + 2 (i % 4), + 1 of rows i / 4 and i / 4 + 8.
template <typename L>
__device__ __forceinline__ void diff_softmax_role(const AttnParams& p, const SeqDev& sq, int pair, int warp, int lane, int n_proc,
                                                  bool backwards, bool all_keys, const int* ktiles, const uint4* keybits,
                                                  uint32_t tmem_base, const uint32_t (&s_full)[2], const uint32_t (&lead_p_full)[2],
                                                  const uint32_t (&o_done)[2], unsigned long long limit, int q_row0, uint8_t* smem) {
  const int t = warp >> 3, h = (warp >> 2) & 1, wq = warp & 3;
  const uint32_t tmem_rows = tmem_base + (static_cast<uint32_t>(wq * 32 + h * 16) << 16);
  const uint32_t tO = tmem_rows + 256 + t * 128;
  constexpr float kBias = 7.0f;                                            // P is held times 2^kBias
  const float c = p.scale_log2;
  float m0 = 0.f, m1 = 0.f, l0 = 0.f, l1 = 0.f;                            // references and (this thread's part of) the sums of its two rows
  bool ok = true, started = false;                                         // started: a key has been seen, m0 and m1 count
  const float lam = diff_lambda(p.diff, pair, lane);

  for (int i = 0; i < n_proc && ok; ++i) {
    const int it = backwards ? n_proc - 1 - i : i;
    const int jt = all_keys ? it : __ldg(&ktiles[it]);
    SOL_DEVICE_CHECK(p.status, jt >= 0 && jt < sq.n_ktiles, kCheckKeyTile);
    uint4 kb = make_uint4(~0u, ~0u, ~0u, ~0u);
    if (!all_keys) kb = __ldg(&keybits[jt]);
    else if (jt == sq.n_ktiles - 1) kb = tail_bits(sq.n_tokens - jt * 128);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t tS = tmem_rows + t * 128 + b * 64;                    // P (32 columns) overwrites the first half of the scores
      const uint32_t bits0 = b ? kb.y : kb.x, bits1 = b ? kb.w : kb.z;
      ok = __all_sync(0xffffffffu, mbar_wait(b ? s_full[1] : s_full[0], i & 1, limit));
      if (!ok) break;
      tc_fence_after();
      uint32_t r[32];                                                      // [4 n], + 1: first row; + 2, + 3: second row
      tmem_ld_16x256b_x8(tS, r);
      tmem_wait_ld_dep32(r);
      if ((bits0 & bits1) != 0xffffffffu) {                                // masked or out-of-range keys get -inf
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if ((((n < 4 ? bits0 : bits1) >> (8 * (n & 3) + 2 * (lane & 3) + e)) & 1u) == 0) {
              r[4 * n + e] = __float_as_uint(-CUDART_INF_F);
              r[4 * n + 2 + e] = __float_as_uint(-CUDART_INF_F);
            }
      }
      auto row_max = [&](int q) {                                          // of row q, over the four threads that share it
        float m = -CUDART_INF_F;
#pragma unroll
        for (int n = 0; n < 8; ++n) m = fmaxf(m, fmaxf(__uint_as_float(r[4 * n + 2 * q]), __uint_as_float(r[4 * n + 2 * q + 1])));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
        return fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
      };
      const bool first = !started && (bits0 | bits1) != 0;                 // the same in all rows: bits are per key
      if (first) {
        m0 = row_max(0);
        m1 = row_max(1);
        started = true;
      }
      float s0, s1;
      auto pass = [&]() {
        const float mc0 = m0 * c - kBias, mc1 = m1 * c - kBias;
        const float2 c2 = make_float2(c, c), n0 = make_float2(-mc0, -mc0), n1 = make_float2(-mc1, -mc1), one = make_float2(1.f, 1.f);
        float2 a0 = make_float2(0.f, 0.f), a1 = a0;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint32_t pk[8];
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const int at = 16 * hf + 4 * n;
            const float2 x0 = fma_f32x2(make_float2(__uint_as_float(r[at]), __uint_as_float(r[at + 1])), c2, n0);
            const float2 x1 = fma_f32x2(make_float2(__uint_as_float(r[at + 2]), __uint_as_float(r[at + 3])), c2, n1);
            const float2 p0 = make_float2(ex2_approx(x0.x), ex2_approx(x0.y)), p1 = make_float2(ex2_approx(x1.x), ex2_approx(x1.y));
            a0 = fma_f32x2(p0, one, a0);
            a1 = fma_f32x2(p1, one, a1);
            pk[2 * n] = pack_f16x2_sat(p0.x, p0.y);
            pk[2 * n + 1] = pack_f16x2_sat(p1.x, p1.y);
          }
          tmem_st_16x128b_x4(tS + 16 * hf, pk);
        }
        s0 = a0.x + a0.y;
        s1 = a1.x + a1.y;
      };
      pass();
      // The pass ran against the current reference maxima, no row maximum taken.  All terms are positive, so sums <= 2^15
      // prove that every term is (fp16 ends at 65504): the references are good enough.  Otherwise, if a row's maximum has
      // grown by more than 2^8, its reference moves, l and O are rescaled and the step is redone before its P is released.
      if (__any_sync(0xffffffffu, !(s0 <= 32768.0f && s1 <= 32768.0f)) && !first) {
        const float x0 = row_max(0), x1 = row_max(1);
        const bool grow0 = (x0 - m0) * c > 8.0f, grow1 = (x1 - m1) * c > 8.0f;
        if (__any_sync(0xffffffffu, grow0 || grow1)) {
          if (lane == 0) atomicAdd(p.counters, 1u);                        // rare path: counted for the tests
          const float f0 = grow0 ? ex2_approx((m0 - x0) * c) : 1.0f, f1 = grow1 ? ex2_approx((m1 - x1) * c) : 1.0f;
          if (grow0) m0 = x0;
          if (grow1) m1 = x1;
          l0 *= f0;
          l1 *= f1;
          ok = __all_sync(0xffffffffu, mbar_wait(b ? o_done[0] : o_done[1], (b ? i : i - 1) & 1, limit));   // the previous step's product is in O
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int cch = 0; cch < 4; ++cch) {
            uint32_t o[16];
            tmem_ld_16x256b_x4(tO + cch * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int n = 0; n < 16; ++n) o[n] = __float_as_uint(__uint_as_float(o[n]) * ((n & 2) ? f1 : f0));
            tmem_st_16x256b_x4(tO + cch * 32, o);
          }
          tmem_wait_st();                                                  // the stale P lands before its replacement
          pass();
        }
      }
      l0 += s0;
      l1 += s1;
      tmem_wait_st();
      tc_fence_before();
      // one arrival per warp, on the leader's barrier (the MMA over both CTAs' rows starts when all sixteen have come)
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(b ? lead_p_full[1] : lead_p_full[0]);
    }
  }

  if (n_proc > 0) {
    // The warps wait for each other in the epilogue, so they must agree on whether it runs: a warp whose wait ran out leaves
    // its mark in its row sums (NaN is what its rows would be) and takes part.
    const uint32_t last = (n_proc - 1) & 1;
    if (ok) ok = __all_sync(0xffffffffu, mbar_wait(o_done[0], last, limit) && mbar_wait(o_done[1], last, limit));
    if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutSoftmax);
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
    l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    if ((lane & 3) == 0) {
      float* xl = reinterpret_cast<float*>(smem + L::kOffXchg) + t * 128 + wq * 32 + h * 16 + (lane >> 2);
      xl[0] = ok ? l0 : CUDART_NAN_F;
      xl[8] = ok ? l1 : CUDART_NAN_F;
    }
    softmax_warps_sync();                                                  // every warp has waited for its own map's products
    tc_fence_after();
    diff_epilogue<L>(p, sq, pair, t, h, q_row0 + wq * 32, lane, wq, tmem_base + (static_cast<uint32_t>(wq * 32) << 16), lam, smem);
  } else {
    // no key tile at all (every key of the sequence masked): the row is defined as zero
    const int qrow = q_row0 + wq * 32 + lane;
    bool store = qrow < sq.n_tokens;
    if (store && p.query_mask != nullptr) store = p.query_mask[sq.tok_start + qrow] != 0;
    if (store) {
      uint8_t* dst = out_row_ptr(p, sq.tok_start + qrow, 2 * pair + t, 2) + h * 64;
#pragma unroll
      for (int c16 = 0; c16 < 4; ++c16) *reinterpret_cast<uint4*>(dst + c16 * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
  }
}

// kDiff: differential attention (head_dim 64, CTA pairs).  The two query tiles of a CTA become the two softmax maps of
// ONE tile of 128 query rows: a head pair (2i, 2i+1) has its two 64-dim Q and K side by side, which in shared memory is
// exactly one 128-dim tile of two 64-column boxes, and map t multiplies box t of Q with box t of K.  Both maps share the
// pair's 128-dim V.
//
// Types: a difference of two maps amplifies their errors, so Q~, K~, P and V are fp16 operands (11 bits instead of 8).  P is
// held times 2^7, so that its range, from 2^15 down to 2^-24, reaches 2^-31 of the reference; four warps turn each V tile from
// bf16 into fp16 in shared memory, in place, tiles ahead of its use, times a power of two that fits fp16's range to the values
// (value_exponent; the product costs 0.6 %).  Error against fp64 at 25,216 tokens: 0.0017, the rounding of the output itself
// (0.0026 with bf16 P and V, 0.0040 with bf16 Q~ and K~ too).
//
// Per key tile and CTA that is 2 x 16384 exponentials (2048 cycles of the special-function unit) against 1536 cycles of
// tensor-core work, so the exponentials bound it.  With the plain kernel's shape (a warp per 32 rows, one score buffer per
// map, one MMA issuer) the unit was busy 58 % of the time: a map waited 1,330 cycles per tile for its scores (P seen, two
// products, scores seen), and a warp alone on its scheduler reached 70 % of the unit's rate.  Hence 64 keys per step and two
// score buffers per map, an issuer per map, and sixteen softmax warps of 16 rows each: a row stays within one warp, whose
// instructions, not the tensor core's latency, are what is left: 2,990 cycles per tile.  25,216 tokens x 20 pairs: 10.35 ms with
// the rotary pass, 943 TFLOP/s, in a long run, where the power limit holds the clock at 1.66 GHz (9.03 ms for a launch of its own).
// Against 10.8 ms with the plain kernel's shape, two threads per row with 64 columns each and the plain kernel's buffers took 11.1
// (the agreement on a row's reference is a barrier per tile), double buffers with eight warps 11.4.
template <int D, int kCtas, bool kDiff = false>
__global__ void __launch_bounds__(kDiff ? kDiffThreads : kAttnThreads, 1)
attn_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const AttnParams p) {
  static_assert(kCtas == 1 || (kCtas == 2 && D == 128), "CTA pairs are built for head_dim 128");
  static_assert(!kDiff || (D == 128 && kCtas == 2), "differential attention runs on CTA pairs, value width 128");
  using L = AttnSmem<D, kCtas, kDiff>;
  constexpr bool kPair = kCtas == 2;
  constexpr int kRows = kDiff ? 128 : 256;              // query rows of one CTA
  constexpr int kTma = kDiff ? 16 : 8, kMma = kTma + 1; // warps: softmax up to here, producer, MMA issuer, others
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t sbase = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - raw_addr);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  // CTA pairs: rank 0 is the leader (issues the MMAs, owns the barriers the other CTA reports to)
  const uint32_t rank = kPair ? cluster_ctarank() : 0u;
  const bool leader = rank == 0;

  const uint32_t sQ = sbase + L::kOffQ;
  const uint32_t sKV = sbase + L::kOffKV;
  const uint32_t bars = sbase + L::kOffBars;
  const uint32_t bar_q_full = bars;
  auto bar_kv_full = [&](int s) { return bars + 8u * (1 + s); };
  auto bar_kv_empty = [&](int s) { return bars + 8u * (1 + L::kStages + s); };
  // (kDiff: [t] and [t + 2] are the two buffers of map t)
  auto bar_s_full = [&](int t) { return bars + 8u * ((t < 2 ? 1 + 2 * L::kStages : 6 + 3 * L::kStages) + t); };
  auto bar_p_full = [&](int t) { return bars + 8u * ((t < 2 ? 3 + 2 * L::kStages : 8 + 3 * L::kStages) + t); };
  auto bar_o_done = [&](int t) { return bars + 8u * ((t < 2 ? 5 + 2 * L::kStages : 10 + 3 * L::kStages) + t); };
  const uint32_t bar_drain = bars + 8u * (7 + 2 * L::kStages);
  const uint32_t bar_drain1 = bars + 8u * (14 + 3 * L::kStages);
  auto bar_v_ready = [&](int s) { return bars + 8u * (8 + 2 * L::kStages + s); };   // kDiff: V of both CTAs is fp16
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(smem + L::kOffTmemPtr);

  // differential attention: the next call's words are larger than this one's, whatever this CTA does below
  if (kDiff && blockIdx.x == 0 && threadIdx.x == 0) atomicAdd(p.value_range, 1ull);
  // ---- which work item (one per CTA, or one per CTA pair)
  const int unit = (int)blockIdx.x / kCtas + p.cta_offset;
  int si = 0;
  // differential attention: 256-row blocks per head PAIR, so the unit counts are half of the single CTAs' (heads is even)
  if (kDiff)      { while (si + 1 < p.n_seqs && unit >= p.seqs[si + 1].work_start / 2) ++si; }
  else if (kPair) { while (si + 1 < p.n_seqs && unit >= p.seqs[si + 1].quad_work_start) ++si; }
  else       { while (si + 1 < p.n_seqs && unit >= p.seqs[si + 1].work_start) ++si; }
  const SeqDev sq = p.seqs[si];
  const int units_per_head = kPair && !kDiff ? (sq.n_qpairs + 1) / 2 : sq.n_qpairs;
  const int local = unit - (kDiff ? sq.work_start / 2 : kPair ? sq.quad_work_start : sq.work_start);
  const int head = local / units_per_head;
  const int blk = local - head * units_per_head;        // query pair (256 rows) or query quad (512 rows); kDiff: head = head pair
  SOL_DEVICE_CHECK(p.status, si < p.n_seqs && local >= 0 && head < p.heads && blk >= 0 && blk < units_per_head, kCheckWorkItem);
  SOL_DEVICE_CHECK(p.status, !(p.fault_inject == 2u && unit == 0), kCheckInjected);
  // a launch may serve a range of heads only (uniform over the CTA / the pair, before any set-up)
  if (head < p.head_begin || head >= p.head_end) return;
  // rectangular mode: a query block without a wanted row has nothing to do (uniform, before any set-up)
  if (p.pair_needed != nullptr) {
    const uint8_t* need = p.pair_needed + sq.pair_start;
    bool any = need[kDiff ? blk : kCtas * blk] != 0;
    if (kPair && !kDiff && 2 * blk + 1 < sq.n_qpairs) any = any || need[2 * blk + 1] != 0;
    if (!any) return;
  }
  // dense: every CTA of a sequence walks the same list of key tiles; block-sparse (single CTAs only): each CTA has its own
  const bool sparse = !kPair && p.cta_list != nullptr;
  const bool all_keys = kDiff && p.keybits == nullptr;  // no mask: no bits and no list were built
  const int n_proc = all_keys ? sq.n_ktiles : sparse ? p.cta_count[unit] : p.ktile_count[si];
  const int* __restrict__ ktiles =
      sparse ? p.cta_list + sq.sparse_list_start + (long long)local * sq.n_ktiles : p.ktile_list + sq.ktile_start;
  const uint4* __restrict__ keybits = p.keybits + sq.ktile_start;
  SOL_DEVICE_CHECK(p.status, n_proc >= 0 && n_proc <= sq.n_ktiles, kCheckTileCount);
  // Successive waves of CTAs walk the key tiles in opposite directions (the softmax does not care about the
  // order): a wave then starts on the tiles its predecessor touched last, which are still in L2, instead of
  // on the ones it touched first, which a long sequence has pushed out by then.
  const bool backwards = ((unit / max(1, p.wave_ctas / kCtas)) & 1) != 0;
  const int q_row0 = blk * (kRows * kCtas) + (int)rank * kRows;   // first local query row of this CTA
  const int tok0 = (int)sq.tok_start;                  // TMA token coordinate of the sequence start
  const unsigned long long limit = p.wait_limit_ns;

  if (warp == kTma && lane == 0) {
    mbar_init(bar_q_full, 1);
    for (int s = 0; s < L::kStages; ++s) {
      mbar_init(bar_kv_full(s), 1);
      mbar_init(bar_kv_empty(s), kDiff ? 2 : 1);         // kDiff: both maps' products have read it
      if (kDiff) mbar_init(bar_v_ready(s), 8);           // four converting warps in either CTA
    }
    for (int t = 0; t < (kDiff ? 4 : 2); ++t) {
      mbar_init(bar_s_full(t), 1);
      mbar_init(bar_p_full(t), (kDiff ? 8 : 4) * kCtas);   // one arrival per softmax warp of the tile, from every CTA
      mbar_init(bar_o_done(t), 1);
    }
    mbar_init(bar_drain, 1);
    if (kDiff) mbar_init(bar_drain1, 1);
    fence_mbar_init();
    prefetch_tensormap(&tm_q);
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
  }
  // A fault recorded by an earlier CTA stops later ones at the door (read once; made uniform over the pair below).
  if (threadIdx.x == 0) tmem_ptr_smem[1] = *reinterpret_cast<volatile unsigned int*>(p.status);
  if (kDiff && warp == kTma + 3 && lane == 0) tmem_ptr_smem[2] = (uint32_t)value_exponent(p.value_range, si, p.heads, head);
  if (warp == kMma) {
    if (kPair) { tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_ptr_smem)), 512); tmem_relinquish_pair(); }
    else       { tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_ptr_smem)), 512); tmem_relinquish(); }
  }
  tc_fence_before();
  if (kPair) cluster_sync_all(); else __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_ptr_smem[0];
  {
    uint32_t stop = tmem_ptr_smem[1];
    if (kPair) {
      // both CTAs must take the same decision: each looks at both flags, and nobody leaves before the other has looked
      stop |= ld_shared_cluster_u32(mapa_shared(smem_u32(const_cast<uint32_t*>(&tmem_ptr_smem[1])), rank ^ 1u));
      cluster_sync_all();
    }
    if (stop != 0) {
      if (warp == kMma) {
        if (kPair) tmem_dealloc_pair(tmem_base, 512); else tmem_dealloc(tmem_base, 512);
      }
      return;
    }
  }
  // barriers of the leader that this CTA reports to (its own when it is the leader)
  const uint32_t lead_q_full = kPair ? mapa_shared(bar_q_full, 0) : bar_q_full;

  if constexpr (kDiff) {
    if (warp < kTma) {
      const int t = warp >> 3;
      const uint32_t s_full[2] = {bar_s_full(t), bar_s_full(t + 2)};
      const uint32_t o_done[2] = {bar_o_done(t), bar_o_done(t + 2)};
      const uint32_t lead_p_full[2] = {mapa_shared(bar_p_full(t), 0), mapa_shared(bar_p_full(t + 2), 0)};
      diff_softmax_role<L>(p, sq, head, warp, lane, n_proc, backwards, all_keys, ktiles, keybits, tmem_base, s_full, lead_p_full,
                           o_done, limit, q_row0, smem);
    }
  } else if (warp < kTma) {
    // =========================================================== softmax / correction / epilogue
    setmaxnreg_inc<SOL_REGS_SOFTMAX>();
    const int t = warp >> 2;
    const int wq = warp & 3;
    const int row = wq * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(wq * 32) << 16;
    const uint32_t tS = tmem_base + lane_off + t * 128;
    const uint32_t tO = tmem_base + lane_off + 256 + t * D;
    const uint32_t lead_p_full = kPair ? mapa_shared(bar_p_full(t), 0) : bar_p_full(t);
    const float c = p.scale_log2;
    float m_ref = -CUDART_INF_F;
    float l = 0.f;
    bool ok = true;

    for (int i = 0; i < n_proc; ++i) {
      const int jt = __ldg(&ktiles[backwards ? n_proc - 1 - i : i]);
      SOL_DEVICE_CHECK(p.status, jt >= 0 && jt < sq.n_ktiles, kCheckKeyTile);
      const uint4 kb = __ldg(&keybits[jt]);
      ok = __all_sync(0xffffffffu, mbar_wait(bar_s_full(t), i & 1, limit));
      if (!ok) break;
      tc_fence_after();

      const bool mixed = (kb.x & kb.y & kb.z & kb.w) != 0xffffffffu;
      uint32_t r[128];
      uint32_t pk[64];
      float tile_sum;
      bool first_half_stored = false;
      if (!mixed && i > 0) {
        // Common case, in two halves: the second half of S is still on its way while the first is exponentiated, and
        // the first half of P is on its way to tensor memory while the second is.
        uint32_t (&r_lo)[64] = *reinterpret_cast<uint32_t(*)[64]>(&r[0]);
        uint32_t (&r_hi)[64] = *reinterpret_cast<uint32_t(*)[64]>(&r[64]);
        tmem_ld32(tS, *reinterpret_cast<uint32_t(*)[32]>(&r[0]));
        tmem_ld32(tS + 32, *reinterpret_cast<uint32_t(*)[32]>(&r[32]));
        tmem_wait_ld_dep64(r_lo);
        tmem_ld32(tS + 64, *reinterpret_cast<uint32_t(*)[32]>(&r[64]));
        tmem_ld32(tS + 96, *reinterpret_cast<uint32_t(*)[32]>(&r[96]));
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        const float mc = m_ref * c;
        softmax_half(r_lo, c, mc, *reinterpret_cast<uint32_t(*)[32]>(&pk[0]), acc);
        tmem_wait_ld_dep64(r_hi);
        tmem_st32(tS, *reinterpret_cast<uint32_t(*)[32]>(&pk[0]));       // columns [0,32): their scores are in registers
        first_half_stored = true;
        softmax_half(r_hi, c, mc, *reinterpret_cast<uint32_t(*)[32]>(&pk[32]), acc);
        tile_sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
      } else {
#pragma unroll
        for (int cch = 0; cch < 4; ++cch) tmem_ld32(tS + cch * 32, *reinterpret_cast<uint32_t(*)[32]>(&r[cch * 32]));
        tmem_wait_ld();
        if (mixed) {
          // masked or out-of-range keys get -inf
#pragma unroll
          for (int cc = 0; cc < 128; ++cc) {
            const uint32_t w = cc < 32 ? kb.x : cc < 64 ? kb.y : cc < 96 ? kb.z : kb.w;
            if (((w >> (cc & 31)) & 1u) == 0) r[cc] = __float_as_uint(-CUDART_INF_F);
          }
        }
        if (i == 0) m_ref = row_max128(r);
        softmax_pass(r, c, m_ref * c, pk, tile_sum);
      }
      // The pass ran against the current reference maximum, no row maximum taken.
      // All terms are positive, so a row sum <= 2^8 proves that every term is <= 2^8: the reference
      // is still good enough (the result does not depend on which reference is used, only overflow
      // does).  Only when the sum is larger (or not finite) is the row maximum computed; if it has grown
      // by more than 2^8 in the exp2 domain the reference moves, l and O are rescaled and the tile is
      // redone from the scores still held in registers, before any of its P is released.  Rare.
      if (__any_sync(0xffffffffu, !(tile_sum <= 256.0f))) {
        const float mx = row_max128(r);
        const bool grow = (mx - m_ref) * c > 8.0f;
        if (__any_sync(0xffffffffu, grow)) {
          if (lane == 0) atomicAdd(p.counters, 1u);                      // rare path: counted for the tests
          const float f = grow ? ex2_approx((m_ref - mx) * c) : 1.0f;
          if (grow) m_ref = mx;
          l *= f;
          ok = __all_sync(0xffffffffu, mbar_wait(bar_o_done(t), (i - 1) & 1, limit));
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int cch = 0; cch < D / 32; ++cch) {
            uint32_t o[32];
            tmem_ld32(tO + cch * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int cc = 0; cc < 32; ++cc) o[cc] = __float_as_uint(__uint_as_float(o[cc]) * f);
            tmem_st32(tO + cch * 32, o);
          }
          softmax_pass(r, c, m_ref * c, pk, tile_sum);
          if (first_half_stored) tmem_wait_st();                         // the stale first half lands before its replacement
          first_half_stored = false;
        }
      }
      l += tile_sum;
      if (!first_half_stored) tmem_st32(tS, *reinterpret_cast<uint32_t(*)[32]>(&pk[0]));
      tmem_st32(tS + 32, *reinterpret_cast<uint32_t(*)[32]>(&pk[32]));
      tmem_wait_st();
      tc_fence_before();
      // one arrival per warp, on the leader's barrier (the MMA over both CTAs' rows starts when all eight have come)
      __syncwarp();
      if (lane == 0) {
        if (kPair) mbar_arrive_cluster(lead_p_full); else mbar_arrive(lead_p_full);
      }
    }

    // ---- epilogue: O / l in the output format, staged through shared memory, coalesced 16-byte stores
    if (ok && n_proc > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait(bar_o_done(t), (n_proc - 1) & 1, limit));
      if (ok) tc_fence_after();
    }
    if (ok && n_proc > 0) {
      const float inv = 1.0f / l;
      uint8_t* stage = smem + L::kOffQ + t * L::kTile + wq * 32 * (D * 2);
      if (p.sink.fmt == kOutInt8)      store_rows_int8<D>(p, sq, head, q_row0 + t * 128 + row, tO, inv);
      else if (p.sink.fmt == kOutE4M3) store_rows<D, true>(p, sq, head, q_row0 + t * 128 + wq * 32, lane, tO, inv, stage);
      else                             store_rows<D, false>(p, sq, head, q_row0 + t * 128 + wq * 32, lane, tO, inv, stage);
    } else if (ok) {
      // no key tile at all (every key of the sequence masked): the row is defined as zero
      const int qrow = q_row0 + t * 128 + row;
      bool store = qrow < sq.n_tokens;
      if (store && p.query_mask != nullptr) store = p.query_mask[sq.tok_start + qrow] != 0;
      if (store && p.sink.fmt == kOutInt8) {
        // a record of zeros: every group's scale code is the smallest one (0x01), as the quantiser writes it
        constexpr int kRecBytes = (D + D / 32 + 15) / 16 * 16;
        uint8_t* dst = out_row_ptr(p, sq.tok_start + qrow, head, 1);
        for (int b = 0; b < kRecBytes; b += 16)
          *reinterpret_cast<uint4*>(dst + b) = make_uint4(b == D ? (D == 128 ? 0x01010101u : 0x00000101u) : 0u, 0u, 0u, 0u);
      } else if (store) {
        const int row_bytes = p.sink.fmt == kOutE4M3 ? D : D * 2;
        uint8_t* dst = out_row_ptr(p, sq.tok_start + qrow, head, row_bytes / D);
        for (int c16 = 0; c16 < row_bytes / 16; ++c16) *reinterpret_cast<uint4*>(dst + c16 * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
    } else if (lane == 0) {
      atomicCAS(p.status, 0u, kStatusTimeoutSoftmax);
    }
  } else {
    setmaxnreg_dec<SOL_REGS_OTHER>();
  }
  if (warp == kTma) {
    // =========================================================== TMA producer
    if (lane == 0) {
      bool ok = true;
      // Q tiles are read once: first to go from L2, so that they do not push out the head's K / V, which every CTA of the
      // head streams.  K / V of a CTA pair are loaded with an evict-last hint on half of the lines: at the high-resolution
      // size that took the DRAM reads of a launch from 6.9 to 5.6 GB (any share from 0.3 to 1.0 did; evict-first on the rest
      // instead of the default: 38-48 GB).  Single CTAs keep the default: there the hint was measured to raise the reads,
      // because the previous heads' tiles then linger.
      const uint64_t pol_once = l2_policy_evict_first();
      const uint64_t pol_kv = l2_policy_evict_last_half();
      // the leader's barrier counts the bytes of both CTAs' loads
      if (leader) mbar_arrive_expect_tx(bar_q_full, kCtas * (kDiff ? 1 : 2) * L::kTile);
      if constexpr (kDiff) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
          tma_load_3d_pair_hint(sQ + hf * L::kHalfBytes, &tm_q, lead_q_full, 0, 2 * head + hf, tok0 + q_row0, pol_once);
      }
#pragma unroll
      for (int t = 0; t < (kDiff ? 0 : 2); ++t)
#pragma unroll
        for (int hf = 0; hf < L::kHalves; ++hf) {
          const uint32_t dst = sQ + t * L::kTile + hf * L::kHalfBytes;
          if (kPair) tma_load_3d_pair_hint(dst, &tm_q, lead_q_full, hf * 64, head, tok0 + q_row0 + t * 128, pol_once);
          else       tma_load_3d_hint(dst, &tm_q, bar_q_full, hf * 64, head, tok0 + q_row0 + t * 128, pol_once);
        }
      uint32_t it = 0, stage = 0, par = 0;
      for (int i = 0; i < n_proc && ok; ++i) {
        const int at = backwards ? n_proc - 1 - i : i;
        const int jt = all_keys ? at : __ldg(&ktiles[at]);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!mbar_wait(bar_kv_empty(stage), par ^ 1u, limit)) { ok = false; break; }
          if (kDiff && kv == 1) mbar_arrive_expect_tx(bar_kv_full(stage), L::kStageBytes);   // V: this CTA's own half, see below
          else if (leader) mbar_arrive_expect_tx(bar_kv_full(stage), L::kTile);
          const uint32_t dst = sKV + stage * L::kStageBytes;
          if (kPair) {
            // this CTA's half of the tile: K = its 64 keys (all head dims, two boxes), V = its 64 head dims (all keys)
            const uint32_t full = mapa_shared(bar_kv_full(stage), 0);
            if (kv == 0) {
#pragma unroll
              for (int hf = 0; hf < L::kHalves; ++hf)
                tma_load_3d_pair_hint(dst + hf * L::kKBoxBytes, &tm_k, full, kDiff ? 0 : hf * 64, kDiff ? 2 * head + hf : head,
                                      tok0 + jt * 128 + (int)rank * 64, pol_kv);
            } else if (kDiff) {
              tma_load_3d_hint(dst, &tm_v, bar_kv_full(stage), 0, 2 * head + (int)rank, tok0 + jt * 128, pol_kv);
            } else {
              tma_load_3d_pair_hint(dst, &tm_v, full, (int)rank * 64, head, tok0 + jt * 128, pol_kv);
            }
          } else {
            const CUtensorMap* tm = kv ? &tm_v : &tm_k;
#pragma unroll
            for (int hf = 0; hf < L::kHalves; ++hf)
              tma_load_3d(dst + hf * L::kHalfBytes, tm, bar_kv_full(stage), hf * 64, head, tok0 + jt * 128);
          }
          ++it;
          if (++stage == (uint32_t)L::kStages) { stage = 0; par ^= 1u; }
        }
      }
      if (!ok) {
        atomicCAS(p.status, 0u, kStatusTimeoutProducer);
        // Let the copies already in flight land before the CTA gives its shared memory back.  A single CTA (and the
        // leader of a pair) can see them on its own barriers; the other CTA of a pair reports to the leader's
        // barriers and cannot, but the wait that just ran out lasted `limit`, far longer than any copy takes.
        if (leader) {
          mbar_wait(bar_q_full, 0, limit);
          const uint32_t first = it > (uint32_t)L::kStages ? it - L::kStages : 0u;
          for (uint32_t j = first; j < it; ++j) mbar_wait(bar_kv_full(j % L::kStages), (j / L::kStages) & 1u, limit);
        } else if (kDiff) {
          const uint32_t first = it > (uint32_t)L::kStages ? it - L::kStages : 0u;
          for (uint32_t j = first | 1u; j < it; j += 2) mbar_wait(bar_kv_full(j % L::kStages), (j / L::kStages) & 1u, limit);
        }
      }
    }
    __syncwarp();
  } else if ((warp == kMma || (kDiff && warp == kMma + 1)) && leader) {
    // =========================================================== MMA issuer
    {
      // The whole warp runs this loop (convergent); one elected lane issues each tcgen05 instruction.
      // differential attention: all operands are fp16, 64 keys at a time
      constexpr uint32_t idesc_qk = kDiff ? idesc_f16_f32(128 * kCtas, 64, false) : idesc_bf16_f32(128 * kCtas, 128, false);
      constexpr uint32_t idesc_pv = kDiff ? idesc_f16_f32(128 * kCtas, D, true) : idesc_bf16_f32(128 * kCtas, D, true);
      bool ok = true;
      const uint32_t v_lbo = p.v_lbo, v_sbo = p.v_sbo;
      // descriptor words: only the low word (address) moves inside the loop
      const uint32_t hi_k = smem_desc_hi_sw128(1024);
      const uint32_t hi_v = smem_desc_hi_sw128(v_sbo);
      const uint32_t q_lo0 = smem_desc_lo(sQ, 16), q_lo1 = smem_desc_lo(sQ + (kDiff ? L::kHalfBytes : L::kTile), 16);
      const uint32_t k_lo_base = smem_desc_lo(sKV, 16);
      const uint32_t v_lo_base = smem_desc_lo(sKV, v_lbo);
      constexpr uint32_t kStageStep = L::kStageBytes >> 4;
      const uint32_t tS0 = tmem_base, tS1 = tmem_base + 128;
      const uint32_t tO0 = tmem_base + 256, tO1 = tmem_base + 256 + D;
      auto commit = [&](uint32_t bar) { if (kPair) tc_commit_elect_pair(bar); else tc_commit_elect(bar); };
      auto wait_full = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, limit); };
      auto issue_qk = [&](uint32_t d_tmem, uint32_t q_lo, uint32_t stage) {
        const uint32_t k_lo = k_lo_base + stage * kStageStep;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t q_off = ((k >> 2) * L::kHalfBytes + (k & 3) * 32) >> 4;
          const uint32_t k_off = ((k >> 2) * L::kKBoxBytes + (k & 3) * 32) >> 4;
          if (kPair) {
            if (k == 0) mma_ss_elect_pair<false>(d_tmem, q_lo + q_off, k_lo + k_off, hi_k, idesc_qk, 0u);
            else        mma_ss_elect_pair<true>(d_tmem, q_lo + q_off, k_lo + k_off, hi_k, idesc_qk, 1u);
          } else {
            if (k == 0) mma_ss_elect<false>(d_tmem, q_lo + q_off, k_lo + k_off, hi_k, idesc_qk, 0u);
            else        mma_ss_elect<true>(d_tmem, q_lo + q_off, k_lo + k_off, hi_k, idesc_qk, 1u);
          }
        }
      };
      auto issue_pv = [&](uint32_t d_tmem, uint32_t p_tmem, uint32_t stage, bool acc) {
        const uint32_t v_lo = v_lo_base + stage * kStageStep;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (kPair) {
            if (k == 0) mma_ts_elect_pair<false>(d_tmem, p_tmem, v_lo, hi_v, idesc_pv, acc ? 1u : 0u);
            else        mma_ts_elect_pair<true>(d_tmem, p_tmem + k * 8, v_lo + k * (2048 >> 4), hi_v, idesc_pv, 1u);
          } else {
            if (k == 0) mma_ts_elect<false>(d_tmem, p_tmem, v_lo, hi_v, idesc_pv, acc ? 1u : 0u);
            else        mma_ts_elect<true>(d_tmem, p_tmem + k * 8, v_lo + k * (2048 >> 4), hi_v, idesc_pv, 1u);
          }
        }
      };
      // consumer position in the K/V ring
      uint32_t st = 0, ph = 0;
      auto advance = [&]() { if (++st == (uint32_t)L::kStages) { st = 0; ph ^= 1u; } };

      if constexpr (kDiff) {
        // One warp per map: what a map waits for does not hold up the other one's products.
        const int t = warp - kMma;
        const uint32_t q_lo = t ? q_lo1 : q_lo0, k_lo_map = k_lo_base + ((t * L::kKBoxBytes) >> 4);
        const uint32_t tS = tmem_base + t * 128, tO = t ? tO1 : tO0;
        // Scores of 64 keys, into buffer b: the map's box of Q and of K, keys 32 b .. + 31 of either CTA's 64.
        auto issue_s = [&](int b, uint32_t stage) {
          const uint32_t k_lo = k_lo_map + stage * kStageStep + b * (4096 >> 4);
          mma_ss_elect_pair<false>(tS + b * 64, q_lo, k_lo, hi_k, idesc_qk, 0u);
#pragma unroll
          for (int k = 1; k < 4; ++k) mma_ss_elect_pair<true>(tS + b * 64, q_lo + k * 2, k_lo + k * 2, hi_k, idesc_qk, 1u);
        };
        auto issue_o = [&](int b, uint32_t stage, bool acc) {
          const uint32_t v_lo = v_lo_base + stage * kStageStep + b * 2 * (2048 >> 4);
          mma_ts_elect_pair<false>(tO, tS + b * 64, v_lo, hi_v, idesc_pv, acc ? 1u : 0u);
#pragma unroll
          for (int k = 1; k < 4; ++k)                                      // keys 32 b + 16 k, then 64 + 32 b + 16 (k - 2)
            mma_ts_elect_pair<true>(tO, tS + b * 64 + k * 8, v_lo + ((k >> 1) * 4 + (k & 1)) * (2048 >> 4), hi_v, idesc_pv, 1u);
        };
        if (n_proc > 0) {
          ok = wait_full(bar_q_full, 0) && wait_full(bar_kv_full(st), ph);
          if (ok) {
            tc_fence_after();
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              issue_s(b, st);
              // (test hook: work item 0 withholds map 1's first signal so that the waits downstream run into their limit)
              if (!(p.fault_inject == 1u && unit == 0 && t == 1 && b == 0)) commit(bar_s_full(t + 2 * b));
            }
            commit(bar_kv_empty(st));
            advance();
          }
          for (int i = 0; i < n_proc && ok; ++i) {
            const uint32_t v_st = st, v_ph = ph;
            advance();
            const bool more = i + 1 < n_proc;
            const uint32_t k_st = st, k_ph = ph;
            if (more) advance();
            if (!wait_full(bar_v_ready(v_st), v_ph)) { ok = false; break; }
            if (more && !wait_full(bar_kv_full(k_st), k_ph)) { ok = false; break; }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              // P of step (i, b) is multiplied, then its place takes the scores of the same half of the next tile, a step before
              // the softmax gets there
              if (!wait_full(bar_p_full(t + 2 * b), i & 1)) { ok = false; break; }
              tc_fence_after();
              issue_o(b, v_st, i > 0 || b > 0);
              commit(bar_o_done(t + 2 * b));
              if (more) {
                issue_s(b, k_st);
                commit(bar_s_full(t + 2 * b));
              }
            }
            if (!ok) break;
            commit(bar_kv_empty(v_st));
            if (more) commit(bar_kv_empty(k_st));
          }
        }
      } else if (n_proc > 0) {
        ok = wait_full(bar_q_full, 0) && wait_full(bar_kv_full(st), ph);
        if (ok) {
          tc_fence_after();
          issue_qk(tS0, q_lo0, st);
          commit(bar_s_full(0));
          issue_qk(tS1, q_lo1, st);
          // (test hook: work item 0 withholds this signal so that the waits downstream run into their limit)
          if (!(p.fault_inject == 1u && unit == 0)) commit(bar_s_full(1));
          commit(bar_kv_empty(st));
          advance();
        }
        for (int i = 0; i < n_proc && ok; ++i) {
          const uint32_t v_st = st, v_ph = ph;
          advance();
          const bool more = i + 1 < n_proc;
          const uint32_t k_st = st, k_ph = ph;
          if (more) advance();
          if (!wait_full(bar_kv_full(v_st), v_ph)) { ok = false; break; }
          if (!wait_full(bar_p_full(0), i & 1)) { ok = false; break; }
          tc_fence_after();
          issue_pv(tO0, tS0, v_st, i > 0);
          commit(bar_o_done(0));
          if (more) {
            if (!wait_full(bar_kv_full(k_st), k_ph)) { ok = false; break; }
            tc_fence_after();
            issue_qk(tS0, q_lo0, k_st);
            commit(bar_s_full(0));
          }
          if (!wait_full(bar_p_full(1), i & 1)) { ok = false; break; }
          tc_fence_after();
          issue_pv(tO1, tS1, v_st, i > 0);
          commit(bar_o_done(1));
          commit(bar_kv_empty(v_st));
          if (more) {
            issue_qk(tS1, q_lo1, k_st);
            commit(bar_s_full(1));
            commit(bar_kv_empty(k_st));
          }
        }
      }
      if (!ok) {
        if (lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutMma);
        // tensor-core work already issued must finish before tensor memory is released (in both CTAs of a pair:
        // the other one learns of it at the cluster barrier below)
        const uint32_t drain = kDiff && warp != kMma ? bar_drain1 : bar_drain;
        commit(drain);
        mbar_wait_warp(drain, 0, limit);
      }
    }
    __syncwarp();
  }

  if (kDiff && warp >= kTma + 4) {
    // =========================================================== V tiles: bf16 -> fp16, in place
    // V tiles are the odd stages of the ring (it has an even number).  Thread = row of this CTA's 128 x 64 half; the chunk
    // order follows the swizzle so that neighbouring rows use different banks.  Rows of keys that do not count become zeros:
    // 0 * (whatever stands there) would not be 0 for infinities and NaN.
    static_assert(!kDiff || L::kStages % 2 == 0, "V tiles keep to the odd stages");
    const int w4 = warp - (kTma + 4), r = w4 * 32 + lane;
    const uint32_t scale2 = (127u - tmem_ptr_smem[2]) * 0x00800080u;       // 2^-v_exp in bf16, twice
    bool ok = true;
    for (int i = 0; i < n_proc && ok; ++i) {
      const int n = 2 * i + 1, stage = n % L::kStages;
      ok = __all_sync(0xffffffffu, mbar_wait(bar_kv_full(stage), (n / L::kStages) & 1, limit));
      if (!ok) break;
      uint8_t* at = smem + L::kOffKV + stage * L::kStageBytes + r * 128;
      const int it = backwards ? n_proc - 1 - i : i;
      const int jt = all_keys ? it : __ldg(&ktiles[it]);
      const uint4 kb = all_keys ? tail_bits(sq.n_tokens - jt * 128) : __ldg(&keybits[jt]);
      const uint32_t bits = w4 == 0 ? kb.x : w4 == 1 ? kb.y : w4 == 2 ? kb.z : kb.w;
      const bool keep = ((bits >> lane) & 1u) != 0;
      uint4 w[8];                                                          // all loads first: they cannot pass the stores
#pragma unroll
      for (int ch = 0; ch < 8; ++ch) w[ch] = *reinterpret_cast<const uint4*>(at + ((ch ^ (r & 7)) << 4));
#pragma unroll
      for (int ch = 0; ch < 8; ++ch) {
        auto half2 = [&](uint32_t x) {                                     // a product with a power of two: exact
          x = mul_bf16x2(x, scale2);
          return pack_f16x2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
        };
        if (!keep) w[ch] = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(at + ((ch ^ (r & 7)) << 4)) = make_uint4(half2(w[ch].x), half2(w[ch].y), half2(w[ch].z), half2(w[ch].w));
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_release(mapa_shared(bar_v_ready(stage), 0));
    }
    if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutProducer);
  }

  // ---- teardown: everyone (of both CTAs) is done with tensor memory and shared memory before they are released
  tc_fence_before();
  if (kPair) cluster_sync_all(); else __syncthreads();
  if (warp == kMma) {
    tc_fence_after();
    if (kPair) tmem_dealloc_pair(tmem_base, 512); else tmem_dealloc(tmem_base, 512);
  }
}

}  // namespace sol
