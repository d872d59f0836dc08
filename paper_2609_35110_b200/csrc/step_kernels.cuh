// Single-token forms: differential attention of one new query token per stream over a K/V cache, and the recurrent step
// of the linear attention.  Both are bound by the bytes they stream (the cache, the state); nothing here is a matrix
// product worth a tensor core: one query row against a cache is 3 multiply-adds per loaded value.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>

#include "attn_fwd_sm100.cuh"
#include "device_types.cuh"
#include "ptx_sm100.cuh"

namespace sol {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ void unpack8(const uint4& w, float (&f)[8]) {
  f[0] = bf16_lo(w.x); f[1] = bf16_hi(w.x); f[2] = bf16_lo(w.y); f[3] = bf16_hi(w.y);
  f[4] = bf16_lo(w.z); f[5] = bf16_hi(w.z); f[6] = bf16_lo(w.w); f[7] = bf16_hi(w.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// ---------------------------------------------------------------------------------------------
// Differential attention, one query token per stream.
//
// Grid: one CTA per (stream, split of the keys, head pair), pairs fastest: neighbouring CTAs read neighbouring parts of
// the same cache rows.  A half-warp owns one key at a time: its 16 lanes hold the 256 bytes of
// the key's pair of K rows (lanes 0-7: map 1, lanes 8-15: map 2) and of the pair's V row, 16 bytes each, so every load
// of a warp covers two whole keys.  A score is a dot product of 8 values per lane and three shuffles over 8 lanes; the
// softmax runs in the log2 domain with a running maximum per half-warp, moved once per batch of kStepKeys keys.  Every
// lane accumulates its 8 value dims for both maps.  Half-warps, then splits, are joined with the usual
// max / rescaled-sum rule in a fixed order, so results do not depend on timing.
//
// Bound by HBM once the instructions per key are few enough: 132 per two keys kept the schedulers 69 % busy and the kernel
// at 222 us for 1.15 GB.  Hence paired fp32 arithmetic, running pointers, a loop without predicates for whole batches, and
// no rescaling of the accumulators while the maximum stands.
// ---------------------------------------------------------------------------------------------
template <bool kValue>
struct Flag { static constexpr bool value = kValue; };

struct DiffStepArgs {
  const __nv_bfloat16* q;
  long long q_row, q_head;               // element strides
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  long long k_slot, k_tok, k_head, v_slot, v_tok, v_head;
  const uint8_t* key_mask;               // [n_slots][capacity] bytes, slot stride mask_slot; nullptr: all
  long long mask_slot;
  const int* lens;
  const int* slots;                      // nullptr: row b uses slot b
  __nv_bfloat16* out;
  long long o_row, o_head;
  int batch, pairs, n_split;
  long long n_slots, capacity;
  float scale_log2;
  DiffWeightsDev w;
  float* partial;                        // [batch][pairs][n_split][kStepPartial] when n_split > 1
};

constexpr int kStepThreads = 256, kStepResident = 3;          // CTAs on an SM (2 and 4 were 15 % slower)
constexpr int kStepKeys = 4;             // keys a half-warp has in flight
constexpr int kStepPartial = 4 + 256;    // m1, m2, l1, l2, then 128 values per map

// (m, l, acc) of two parts -> their union; a part without keys has m = -inf and counts for nothing.  A part whose keys all have
// a score of -infinity has m = -kStepLowest and l = 0: beside others it counts for nothing too, on its own it gives 0 / 0.
constexpr float kStepLowest = 3.402823466e38f;
__device__ __forceinline__ float part_weight(float m, float m_all) { return m == -CUDART_INF_F ? 0.f : exp2f(m - m_all); }

// out rows of one (stream, pair) from the joined maps: thread e < 128 holds value e of the difference x.  A row without a
// key (empty, the same in all threads) is zeros, with no lambda and no norm: 0 * infinity and 0 / sqrt(0) are not 0.
__device__ __forceinline__ void diff_step_finish(const DiffStepArgs& a, int b, int pair, int e, float x, bool empty, float* red) {
  if (empty) x = 0.f;
  if (a.w.gain != nullptr && !empty) {
    float ss = x * x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if ((e & 31) == 0) red[e >> 5] = ss;
    asm volatile("bar.sync 2, 128;" ::: "memory");
    ss = (red[0] + red[1]) + (red[2] + red[3]);
    if (ss > 1e-30f && ss < 1e30f) {
      x *= (1.0f - a.w.lambda_init) / sqrtf(ss * (1.0f / 128.0f) + a.w.eps) * __ldg(a.w.gain + e);
    } else {                                               // rare: squares beyond fp32's range (the same in all threads)
      __shared__ double wide[4];
      double sq = (double)x * x;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
      if ((e & 31) == 0) wide[e >> 5] = sq;
      asm volatile("bar.sync 2, 128;" ::: "memory");
      sq = (wide[0] + wide[1]) + (wide[2] + wide[3]);
      x = (float)((1.0 - (double)a.w.lambda_init) * x / sqrt(sq * (1.0 / 128.0) + (double)a.w.eps)) * __ldg(a.w.gain + e);
    }
  }
  a.out[(long long)b * a.o_row + (long long)(2 * pair + (e >> 6)) * a.o_head + (e & 63)] = __float2bfloat16_rn(x);
}

__global__ void __launch_bounds__(kStepThreads, kStepResident) diff_step_kernel(const DiffStepArgs a) {
  __shared__ float s_m[2][16], s_l[2][16];
  __shared__ float s_acc[2][16][128];
  __shared__ float s_red[4];
  const int pair = blockIdx.x % a.pairs, split = blockIdx.x / a.pairs % a.n_split, b = blockIdx.x / a.pairs / a.n_split;
  const long long slot = a.slots != nullptr ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) return;                      // idle row: left as it is
  const long long len = max(0ll, min((long long)a.lens[b], a.capacity));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15, map = l16 >> 3;
  // keys of this split: equal contiguous ranges, none for the last splits of a short stream
  const long long per = max((len + a.n_split - 1) / a.n_split, 16ll * kStepKeys);
  const long long k0 = min(len, split * per), k1 = min(len, k0 + per);

  // lane l16 of a half-warp: head 2 * pair + map, dims 8 * (l16 & 7) .. + 7, for Q, K and V alike
  const int head = 2 * pair + map, d0 = (l16 & 7) * 8;
  float2 q[4];
  {
    float f[8];
    unpack8(*reinterpret_cast<const uint4*>(a.q + (long long)b * a.q_row + (long long)head * a.q_head + d0), f);
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = make_float2(f[2 * i] * a.scale_log2, f[2 * i + 1] * a.scale_log2);
  }
  const __nv_bfloat16* kp = a.k + slot * a.k_slot + (long long)head * a.k_head + d0;
  const __nv_bfloat16* vp = a.v + slot * a.v_slot + (long long)head * a.v_head + d0;
  const uint8_t* mp = a.key_mask != nullptr ? a.key_mask + slot * a.mask_slot : nullptr;

  float m = -CUDART_INF_F, l = 0.f;      // of this lane's own map
  bool seen = false;                     // this half-warp has had a valid key
  float2 acc0[4] = {}, acc1[4] = {};     // this lane's value dims, map 1 and map 2
  const int hw = warp * 2 + half;        // 16 half-warps
  const __nv_bfloat16* kc = kp + (k0 + hw) * a.k_tok;                      // this half-warp's next key
  const __nv_bfloat16* vc = vp + (k0 + hw) * a.v_tok;
  const long long k_step = 16 * a.k_tok, v_step = 16 * a.v_tok;
  // a batch of keys first, first + 16, ...; kWhole: all of them exist
  auto batch = [&](long long first, auto whole, auto masked) {
    constexpr bool kWhole = decltype(whole)::value, kMasked = decltype(masked)::value;
    uint4 kw[kStepKeys], vw[kStepKeys];
    bool on[kStepKeys];
#pragma unroll
    for (int u = 0; u < kStepKeys; ++u) {
      on[u] = kWhole || first + u * 16 < k1;
      kw[u] = on[u] ? __ldg(reinterpret_cast<const uint4*>(kc)) : make_uint4(0, 0, 0, 0);
      vw[u] = on[u] ? __ldg(reinterpret_cast<const uint4*>(vc)) : make_uint4(0, 0, 0, 0);
      kc += k_step;
      vc += v_step;
      if (kMasked && on[u]) on[u] = __ldg(mp + first + u * 16) != 0;
      seen = seen || on[u];
    }
    if (kMasked) {
      // a masked key has score -inf and value 0: whatever the cache holds there, infinities and NaN included, has no effect
#pragma unroll
      for (int u = 0; u < kStepKeys; ++u)
        if (!on[u]) vw[u] = make_uint4(0, 0, 0, 0);
    }
    float s[kStepKeys];
    float mx = m;
#pragma unroll
    for (int u = 0; u < kStepKeys; ++u) {
      const uint32_t w[4] = {kw[u].x, kw[u].y, kw[u].z, kw[u].w};
      float2 d2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) d2 = fma_f32x2(q[i], make_float2(bf16_lo(w[i]), bf16_hi(w[i])), d2);
      float d = d2.x + d2.y;
      d += __shfl_xor_sync(0xffffffffu, d, 1);
      d += __shfl_xor_sync(0xffffffffu, d, 2);
      d += __shfl_xor_sync(0xffffffffu, d, 4);
      s[u] = (kWhole && !kMasked) || on[u] ? d : -CUDART_INF_F;
      mx = fmaxf(mx, s[u]);
    }
    if (__any_sync(0xffffffffu, mx > m)) {
      const float f_old = mx > m ? ex2_approx(m - mx) : 1.f;
      m = mx;
      l *= f_old;
      const float f_other = __shfl_xor_sync(0xffffffffu, f_old, 8);
      const float g0 = map ? f_other : f_old, g1 = map ? f_old : f_other;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc0[i] = mul_f32x2(acc0[i], make_float2(g0, g0));
        acc1[i] = mul_f32x2(acc1[i], make_float2(g1, g1));
      }
    }
    const float ref = m == -CUDART_INF_F ? 0.f : m;                        // no key yet: every exponential below is 2^-inf = 0
#pragma unroll
    for (int u = 0; u < kStepKeys; ++u) {
      const float p = ex2_approx(s[u] - ref);
      l += p;
      const float p_other = __shfl_xor_sync(0xffffffffu, p, 8);
      const float p0 = map ? p_other : p, p1 = map ? p : p_other;
      const uint32_t w[4] = {vw[u].x, vw[u].y, vw[u].z, vw[u].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v2 = make_float2(bf16_lo(w[i]), bf16_hi(w[i]));
        acc0[i] = fma_f32x2(make_float2(p0, p0), v2, acc0[i]);
        acc1[i] = fma_f32x2(make_float2(p1, p1), v2, acc1[i]);
      }
    }
  };
  long long base = k0;
  if (mp == nullptr) {
#pragma unroll 1
    for (; base + 16 * kStepKeys <= k1; base += 16 * kStepKeys) batch(base + hw, Flag<true>{}, Flag<false>{});
    if (base < k1) batch(base + hw, Flag<false>{}, Flag<false>{});
  } else {
#pragma unroll 1
    for (; base + 16 * kStepKeys <= k1; base += 16 * kStepKeys) batch(base + hw, Flag<true>{}, Flag<true>{});
    if (base < k1) batch(base + hw, Flag<false>{}, Flag<true>{});
  }
  if (seen) m = fmaxf(m, -kStepLowest);
  if ((l16 & 7) == 0) { s_m[map][hw] = m; s_l[map][hw] = l; }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    *reinterpret_cast<float2*>(&s_acc[0][hw][l16 * 8 + 2 * i]) = acc0[i];
    *reinterpret_cast<float2*>(&s_acc[1][hw][l16 * 8 + 2 * i]) = acc1[i];
  }
  __syncthreads();
  if (threadIdx.x >= 128) return;
  const int e = threadIdx.x;
  float mm[2], ll[2], xx[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    float top = -CUDART_INF_F;
    for (int h = 0; h < 16; ++h) top = fmaxf(top, s_m[t][h]);
    float sl = 0.f, sx = 0.f;
    for (int h = 0; h < 16; ++h) {
      const float w = part_weight(s_m[t][h], top);
      sl = fmaf(w, s_l[t][h], sl);
      sx = fmaf(w, s_acc[t][h][e], sx);
    }
    mm[t] = top; ll[t] = sl; xx[t] = sx;
  }
  if (a.n_split > 1) {
    float* dst = a.partial + (((long long)b * a.pairs + pair) * a.n_split + split) * kStepPartial;
    if (e == 0) { dst[0] = mm[0]; dst[1] = mm[1]; dst[2] = ll[0]; dst[3] = ll[1]; }
    dst[4 + e] = xx[0];
    dst[4 + 128 + e] = xx[1];
    return;
  }
  const float lam = diff_lambda(a.w, pair, e & 31);
  diff_step_finish(a, b, pair, e, xx[0] / ll[0] - lam * (xx[1] / ll[1]), mm[0] == -CUDART_INF_F, s_red);
}

// Joins the splits of one (stream, pair): thread = one value of one map.  The weights of the splits are formed once, in
// parallel, and the values are summed with eight loads in flight: a loop over dependent loads took longer than a tenth of
// the whole call.
constexpr int kStepMaxSplit = 512;
__global__ void __launch_bounds__(256) diff_step_join_kernel(const DiffStepArgs a) {
  __shared__ float s_w[2][kStepMaxSplit];
  __shared__ float s_top[8], s_sum[8], s_x[128], s_red[4];
  const int pair = blockIdx.x % a.pairs, b = blockIdx.x / a.pairs, t = threadIdx.x >> 7, e = threadIdx.x & 127;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long slot = a.slots != nullptr ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) return;
  const float* src = a.partial + ((long long)b * a.pairs + pair) * a.n_split * kStepPartial;
  float top = -CUDART_INF_F;
  for (int s = e; s < a.n_split; s += 128) top = fmaxf(top, src[(long long)s * kStepPartial + t]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
  top = fmaxf(fmaxf(s_top[4 * t], s_top[4 * t + 1]), fmaxf(s_top[4 * t + 2], s_top[4 * t + 3]));
  float sl = 0.f;
  for (int s = e; s < a.n_split; s += 128) {
    const float w = part_weight(src[(long long)s * kStepPartial + t], top);
    s_w[t][s] = w;
    sl = fmaf(w, src[(long long)s * kStepPartial + 2 + t], sl);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sl += __shfl_xor_sync(0xffffffffu, sl, o);
  if (lane == 0) s_sum[warp] = sl;
  __syncthreads();
  sl = (s_sum[4 * t] + s_sum[4 * t + 1]) + (s_sum[4 * t + 2] + s_sum[4 * t + 3]);
  float x = 0.f;
  const float* val = src + 4 + t * 128 + e;
#pragma unroll 8
  for (int s = 0; s < a.n_split; ++s) x = fmaf(s_w[t][s], val[(long long)s * kStepPartial], x);
  x /= sl;                                                                 // 0 / 0 without a key, in both maps
  if (t == 1) s_x[e] = x;
  __syncthreads();
  if (t == 1) return;
  const float lam = diff_lambda(a.w, pair, lane);
  diff_step_finish(a, b, pair, e, x - lam * s_x[e], top == -CUDART_INF_F, s_red);
}

// ---------------------------------------------------------------------------------------------
// Linear attention, one token per row: S' = exp(log_decay) S + k^T v, o = scale * q S'.
//
// One CTA = one (row, head, 32 columns of the state): columns are independent of each other in both formulas, so a
// state splits into slices without any join, and a slice of 128 x 32 fp32 is one round of 16-byte loads of 128 threads
// (8 per thread, all in flight at once).  Lane layout: 8 lanes cover a 128-byte row slice, a warp covers 4 rows per
// load.  Bound by reading and writing the state once.
//
// Rows that name the same slot are successive tokens of that stream: the CTA of the first such row walks over them in
// row order with the state in registers, the others leave.
// ---------------------------------------------------------------------------------------------
struct LinearStepArgs {
  const __nv_bfloat16* x[3];             // q, k, v
  long long row[3], head[3];             // element strides
  __nv_bfloat16* out;
  long long o_row, o_head;
  const float* log_decay;
  float scale;
  const float* state_in;                 // [n_slots][heads][D][D]; may equal state_out
  float* state_out;
  const int* slots;                      // nullptr: row b uses slot b
  int batch, heads;
  long long n_slots;
};

template <int D>
__global__ void __launch_bounds__(128) linear_step_kernel(const LinearStepArgs a) {
  constexpr int kSlices = D / 32, kRows = D / 16;        // state rows per thread
  __shared__ float s_q[D], s_k[D];
  __shared__ float s_o[4][32];
  __shared__ int s_next;
  const int slice = blockIdx.x % kSlices;
  const long long item = blockIdx.x / kSlices;
  const int head = (int)(item % a.heads);
  int b = (int)(item / a.heads);
  const long long slot = a.slots != nullptr ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) return;             // idle row: left as it is, and so is every state
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int r0 = warp * 4 + (lane >> 3), c0 = (lane & 7) * 4;             // rows r0 + 16 i, columns c0 .. c0 + 3 of the slice
  const long long base = (slot * a.heads + head) * (long long)(D * D) + slice * 32 + c0;
  float4 S[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) S[i] = *reinterpret_cast<const float4*>(a.state_in + base + (long long)(r0 + 16 * i) * D);
  // who walks this slot: the first row that names it; which row comes next
  bool earlier = false;
  if (a.slots != nullptr) {
    if (tid == 0) s_next = a.batch;
    __syncthreads();
    for (int i = tid; i < a.batch; i += 128)
      if (i != b && a.slots[i] == (int)slot) {
        if (i < b) earlier = true;
        else atomicMin(&s_next, i);
      }
    if (__syncthreads_or(earlier)) return;
  }
  const float log_decay = a.log_decay[head];
  const float g = expf(log_decay > 0.f ? 0.f : log_decay);                // NaN stays NaN
  if (g == 0.f) {                                        // forgets whatever the state holds: 0 * infinity would be NaN
#pragma unroll
    for (int i = 0; i < kRows; ++i) S[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  while (true) {
    if (tid < D) {
      s_q[tid] = __bfloat162float(a.x[0][(long long)b * a.row[0] + (long long)head * a.head[0] + tid]);
      s_k[tid] = __bfloat162float(a.x[1][(long long)b * a.row[1] + (long long)head * a.head[1] + tid]);
    }
    const uint2 vw = *reinterpret_cast<const uint2*>(a.x[2] + (long long)b * a.row[2] + (long long)head * a.head[2] + slice * 32 + c0);
    const float4 v = make_float4(bf16_lo(vw.x), bf16_hi(vw.x), bf16_lo(vw.y), bf16_hi(vw.y));
    __syncthreads();
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const float k = s_k[r0 + 16 * i], q = s_q[r0 + 16 * i];
      S[i].x = fmaf(k, v.x, g * S[i].x); S[i].y = fmaf(k, v.y, g * S[i].y);
      S[i].z = fmaf(k, v.z, g * S[i].z); S[i].w = fmaf(k, v.w, g * S[i].w);
      o.x = fmaf(q, S[i].x, o.x); o.y = fmaf(q, S[i].y, o.y); o.z = fmaf(q, S[i].z, o.z); o.w = fmaf(q, S[i].w, o.w);
    }
#pragma unroll
    for (int d = 8; d < 32; d <<= 1) {
      o.x += __shfl_xor_sync(0xffffffffu, o.x, d); o.y += __shfl_xor_sync(0xffffffffu, o.y, d);
      o.z += __shfl_xor_sync(0xffffffffu, o.z, d); o.w += __shfl_xor_sync(0xffffffffu, o.w, d);
    }
    if (lane < 8) *reinterpret_cast<float4*>(&s_o[warp][c0]) = o;
    __syncthreads();
    if (tid < 32)
      a.out[(long long)b * a.o_row + (long long)head * a.o_head + slice * 32 + tid] =
          __float2bfloat16_rn(a.scale * ((s_o[0][tid] + s_o[1][tid]) + (s_o[2][tid] + s_o[3][tid])));
    const int next = a.slots != nullptr ? s_next : a.batch;
    if (next >= a.batch) break;
    b = next;
    __syncthreads();
    if (tid == 0) s_next = a.batch;
    __syncthreads();
    for (int i = b + 1 + tid; i < a.batch; i += 128)
      if (a.slots[i] == (int)slot) atomicMin(&s_next, i);
    // (the barrier inside the next round orders these minima before s_next is read again)
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) *reinterpret_cast<float4*>(a.state_out + base + (long long)(r0 + 16 * i) * D) = S[i];
}

}  // namespace sol
