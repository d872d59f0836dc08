// Attention of many query rows over keys and values that live in the pages of a cache or in an encoder's states: tcgen05 tensor
// cores, accumulators in tensor memory, online softmax in registers.  The two query tiles of a CTA ping-pong as in
// attn_fwd_sm100.cuh; what differs is what surrounds them.
//
// A tile is 128 (token, head) rows of one K/V head: 128 / group tokens x the group's heads, head fastest, which one TMA box brings
// side by side; so grouped heads share every K and V tile.  A unit is two such tiles, one K/V head and a range of key tiles (all of
// them, or a part when there are few units; the parts are joined by join_units_kernel).
//
// CTAs are persistent, one per SM, and take units from a counter, so that short contexts do not pay for a CTA's start (tensor
// memory, barriers, the first loads) and its last stores per unit, and streams of different length even out.  A warp looks the
// next unit up while the present one is computed: its Q, K and V are on their way, and its first scores are computed, while the
// softmax warps still write the last one's rows.
//   warps 0-3, 4-7  softmax and epilogue of tile 0, tile 1 (thread = row)
//   warp 8          loads: Q by one box per tile half; K and V pages by one box per page part and half, a lane each
//   warp 9          tcgen05.mma issuer
//   warp 10         takes units
//   warp 11         values of keys that do not count become zeros in shared memory (0 * NaN would not be 0)
// Tensor memory: S0 | S1 | O0 | O1 as in attn_fwd_sm100.cuh.
//
// Rounding: S, the running sums and O are fp32; P is rounded to bf16, the type of V, for its product (half a step of every term: 0.0023
// relative error against 0.0017 of the output's own rounding).  A second bf16 part of P, as in few_rows_kernel, would be another
// product per key tile and twice P's way through tensor memory, on the chain that bounds the kernel.
//
// What bounds it is that chain, scores -> softmax -> P -> product of two tiles in turn: 3,650 cycles per 128 keys, as in the dense kernel;
// the tensor pipe works 40 to 55 % of that, the exponentials as much.  In ten calls after a pause, and in a run of seconds (clocks under
// the 1 kW cap): 4,680 rows x 40 heads x 128 over 25,216 keys 1.94 ms (1.25 PFLOP/s) and 2.25 to 2.33; 60 tokens x 40 / 8 heads over
// 111,856 keys 208 us and 231 to 238 (the second tile's place is empty in half of the units); 25,216 rows x 40 heads over 512 states 269
// and 311 to 322, of which some 5,000 cycles per unit and four key tiles are its start and end, of both tiles at the same time.  No gain: packed pairs of
// fp32 operations, a polynomial for an eighth to a third of the exponentials (2 to 5 % slower), one MMA issuer per tile (a quarter slower).
#pragma once
#include "attn_fwd_sm100.cuh"
#include "context_attn.cuh"

namespace sol {

struct UnitDev {
  Span span;
  long long tok0;               // first token of the sequence in the packed tensors
  long long part;               // index of this unit's partial rows, or -1: the rows themselves are written
  int t0, n_tok;                // first new token of the unit; new tokens of the sequence
  int kv_head;
  int tile_begin, n_keys;       // key tiles: the first one (where all are taken), how many
  uint32_t live;                // with a mask and no more than 32 key tiles: those that hold a valid key; else 0
  int n_tiles;                  // query tiles: 1 or 2
  int lim[2];                   // keys below lim[t] count for every row of tile t
  int last;                     // no more units
  int withhold;                 // test hook: "the scores of the last tile are there" is not said
};

struct ContextParams {
  QueriesDev a;
  KeysDev d;
  // Up to kSortedSeqs sequences are planned on the device, where their keys are known, into at most max_parts parts of split units.
  int max_parts;
  // More sequences: row units per K/V head, numbered with room for empty ones (find_sequence); all heads' units, of which the first
  // n_whole take all of their keys and the others' keys are split.
  long long units, n_whole, n_tail;
  int n_split;
  int tok_per_tile;             // 128 / group
  unsigned int inv_group;       // ceil(2^16 / group): x / group = x * inv_group >> 16 for x < 128
  int box_rows;                 // tokens of a K/V box: a power of two that divides the page size, at most 128
  float* partial;               // [part][2 * tok_per_tile * group][D + 4]
  JoinUnit* join;               // whose rows the parts hold, a unit each
  int* join_count;
  unsigned int* counter;        // next unit; 0 between launches
  unsigned int* status;
  unsigned int* rescales;
  unsigned long long wait_limit_ns;
  unsigned int fault_inject;    // 1: item 0 withholds "the scores of the last tile are there"
  unsigned int v_lbo, v_sbo;
};

// Up to so many sequences are planned on the device: taken in the order of their keys, most first, so that long units do not come
// last, and their keys split where that evens the work out.
constexpr int kSortedSeqs = 32;
constexpr int kPlanSms = 148;
// What a unit needs to know of its sequence, looked up once.
struct SeqNote {
  int at;                       // stream, or first row of the context
  int n, cap;                   // as in Span; n < 0: idle
  int tok0, n_tok;              // first token in the packed tensors; new tokens
};
constexpr int kUnitRing = 4, kNear = 6;

template <int D>
struct ContextSmem {
  static constexpr int kTile = 128 * D * 2;
  static constexpr int kHalves = D / 64;
  static constexpr int kHalfBytes = 128 * 128;
  static constexpr int kStages = D == 128 ? 4 : 9;       // K and V tiles alternate
  static constexpr int kVRing = 8;                        // "V is clean" barriers: more than V tiles fit the ring
  static constexpr int kOffQ = 0;
  static constexpr int kOffKV = 2 * kTile;
  static constexpr int kOffStage = kOffKV + kStages * kTile;   // 4 KB per softmax warp
  static constexpr int kOffBars = kOffStage + 8 * 4096;
  static constexpr int kNumBars = 2 * kStages + 4 + 6 + 3 * kUnitRing + kVRing + 1;
  static constexpr int kOffTmemPtr = kOffBars + kNumBars * 8;
  static constexpr int kOffUnits = (kOffTmemPtr + 16 + 15) / 16 * 16;
  static constexpr int kOffOrder = kOffUnits + kUnitRing * (int)sizeof(UnitDev);   // sequence, first item, units, parts, first part: kSortedSeqs each
  static constexpr int kOffSeqs = kOffOrder + 5 * kSortedSeqs * 4;
  static constexpr int kBytes = kOffSeqs + kSortedSeqs * (int)sizeof(SeqNote);
  static constexpr int kDynBytes = kBytes + 1024;
  static_assert(kDynBytes <= 227 * 1024, "what a CTA may have");
};

// A unit's key tiles, one after another.
template <bool kMask>
struct TileWalk {
  int jt, left;
  uint32_t live;
  __device__ __forceinline__ explicit TileWalk(const UnitDev& un) : jt(un.tile_begin), left(un.n_keys), live(kMask ? un.live : 0u) {
    if (kMask && live != 0) jt = __ffs(live) - 1;
  }
  __device__ __forceinline__ bool more() const { return left > 0; }
  __device__ __forceinline__ void next() {
    --left;
    if (kMask && live != 0) {
      live &= live - 1;
      jt = __ffs(live) - 1;
    } else {
      ++jt;
    }
  }
};

// Validity of 32 keys from `first` on: those below `limit`.
__device__ __forceinline__ uint32_t below(int limit, int first) {
  const int n = limit - first;
  return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
}

// kBoxes: rows are written by TMA boxes; for contexts, where 32 is a multiple of the heads per K/V head.  (Short contexts have many
// epilogues; in the masked paged kernel the registers for it cost more than it gave: four streams by frames 324 and 336 us.)
template <int D, bool kPaged, bool kMask, bool kBoxes>
__global__ void __launch_bounds__(kAttnThreads, 1)
context_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                    const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o, const __grid_constant__ ContextParams p) {
  using L = ContextSmem<D>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t sbase = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - raw_addr);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  const uint32_t sQ = sbase + L::kOffQ, sKV = sbase + L::kOffKV, bars = sbase + L::kOffBars;
  auto bar_kv_full = [&](int s) { return bars + 8u * s; };
  auto bar_kv_empty = [&](int s) { return bars + 8u * (L::kStages + s); };
  constexpr int kB = 2 * L::kStages;
  auto bar_q_full = [&](int t) { return bars + 8u * (kB + t); };
  auto bar_q_empty = [&](int t) { return bars + 8u * (kB + 2 + t); };
  auto bar_s_full = [&](int t) { return bars + 8u * (kB + 4 + t); };
  auto bar_p_full = [&](int t) { return bars + 8u * (kB + 6 + t); };
  auto bar_o_done = [&](int t) { return bars + 8u * (kB + 8 + t); };
  auto bar_u_full = [&](uint32_t u) { return bars + 8u * (kB + 10 + (u & (kUnitRing - 1))); };
  auto bar_u_empty = [&](uint32_t u) { return bars + 8u * (kB + 10 + kUnitRing + (u & (kUnitRing - 1))); };
  auto bar_v_clean = [&](uint32_t n) { return bars + 8u * (kB + 10 + 2 * kUnitRing + (n & (L::kVRing - 1))); };
  const uint32_t bar_drain = bars + 8u * (kB + 10 + 2 * kUnitRing + L::kVRing);
  auto bar_near = [&](uint32_t u) { return bars + 8u * (kB + 11 + 2 * kUnitRing + L::kVRing + (u & (kUnitRing - 1))); };
  auto round_of = [](uint32_t u) { return (u / kUnitRing) & 1u; };
  volatile uint32_t* tmem_ptr_smem = reinterpret_cast<volatile uint32_t*>(smem + L::kOffTmemPtr);
  UnitDev* units = reinterpret_cast<UnitDev*>(smem + L::kOffUnits);
  const unsigned long long limit = p.wait_limit_ns;

  chained_wait();
  chained_next();
  if (warp == 8 && lane == 0) {
    for (int s = 0; s < L::kStages; ++s) { mbar_init(bar_kv_full(s), 1); mbar_init(bar_kv_empty(s), 1); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(bar_q_full(t), 1);
      mbar_init(bar_q_empty(t), 1);
      mbar_init(bar_s_full(t), 1);
      mbar_init(bar_p_full(t), 4);
      mbar_init(bar_o_done(t), 1);
    }
    for (int u = 0; u < kUnitRing; ++u) {
      mbar_init(bar_u_full(u), 1);
      mbar_init(bar_near(u), 1);                           // the loads of a unit are almost through
      mbar_init(bar_u_empty(u), 11);                       // eight softmax warps, loads, issuer, cleaner
    }
    for (int n = 0; n < L::kVRing; ++n) mbar_init(bar_v_clean(n), 1);
    mbar_init(bar_drain, 1);
    fence_mbar_init();
    prefetch_tensormap(&tm_q);
    prefetch_tensormap(&tm_k);
    prefetch_tensormap(&tm_v);
    if (kBoxes) prefetch_tensormap(&tm_o);
  }
  if (threadIdx.x == 0) tmem_ptr_smem[1] = *reinterpret_cast<volatile unsigned int*>(p.status);
  if (warp == 9) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_ptr_smem)), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_ptr_smem[0];
  if (tmem_ptr_smem[1] != 0) {                             // a fault was recorded earlier: nothing starts any more
    if (warp == 9) tmem_dealloc(tmem_base, 512);
    return;
  }
  // A role that is not part of a unit, or far ahead, waits for as long as the unit takes: it gives up once a wait somewhere else
  // has run out, or after 64 limits.
  auto wait_long = [&](uint32_t bar, uint32_t parity) {
    for (int n = 0; n < 64; ++n) {
      if (mbar_wait_warp(bar, parity, limit)) return true;
      if (*reinterpret_cast<volatile unsigned int*>(p.status) != 0) return false;
    }
    return false;
  };
  auto release_unit = [&](uint32_t u) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_u_empty(u));
  };

  if (warp < 8) {
    // =========================================================== softmax / epilogue
    setmaxnreg_inc<SOL_REGS_SOFTMAX>();
    const int t = warp >> 2, wq = warp & 3, row = wq * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(wq * 32) << 16;
    const uint32_t tS = tmem_base + lane_off + t * 128;
    const uint32_t tO = tmem_base + lane_off + 256 + t * D;
    const float c = p.a.scale_log2;
    const int group = p.a.group;
    const int tile_rows = p.tok_per_tile * group;
    uint32_t n_s = 0;                                      // key tiles of this query tile so far
    bool ok = true;
    // Sequences without any key have no units (where they are sorted): their rows are zeros, which all CTAs write together.
    if (p.a.n_seqs <= kSortedSeqs) {
      bool empty = false;
      if (lane < p.a.n_seqs) {
        const Span sp = find_span<kPaged>(p.d, p.a.seqs[lane].seq_id);
        empty = !sp.idle && sp.n == 0;
      }
      for (unsigned which = __ballot_sync(0xffffffffu, empty); which != 0; which &= which - 1) {
        const SeqDev& sq = p.a.seqs[__ffs(which) - 1];
        const int chunks = p.d.c.kv_heads * group * (D / 8);
        for (long long tok = (long long)blockIdx.x * 8 + warp; tok < sq.n_tokens; tok += (long long)gridDim.x * 8) {
          __nv_bfloat16* dst = p.a.out + (sq.tok_start + tok) * p.a.o_tok;
          for (int x = lane; x < chunks; x += 32)
            *reinterpret_cast<uint4*>(dst + (long long)(x / (D / 8)) * p.a.o_head + x % (D / 8) * 8) = make_uint4(0u, 0u, 0u, 0u);
        }
      }
    }
    for (uint32_t u = 0;; ++u) {
      if (!wait_long(bar_u_full(u), round_of(u))) { ok = false; break; }
      const UnitDev& un = units[u & (kUnitRing - 1)];
      if (un.last) break;
      if (t >= un.n_tiles) { release_unit(u); continue; }
      const int lim_all = un.lim[t];
      const bool any_keys = un.n_keys > 0;
      const uint8_t* mask = kMask ? un.span.mask : nullptr;
      const int cap = un.span.cap;
      const int tok = un.t0 + t * p.tok_per_tile + (int)(row * p.inv_group >> 16);       // this thread's new token
      const bool mine = row < tile_rows && tok < un.n_tok;
      const int lim = mine ? key_limit(un.span, un.n_tok, tok, p.a.causal) : 0x7fffffff;
      float m_ref = -CUDART_INF_F, l = 0.f;
      bool seen = false, started = false;                  // started: every row of the warp has its reference
      uint32_t next_mask = 0;                              // mask bytes of the next key tile: keys lane, + 32, + 64, + 96
      auto fetch_mask = [&](int jt) {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = jt * 128 + e * 32 + lane;
          if (key < cap && mask[key] != 0) w |= 1u << e;
        }
        return w;
      };
      TileWalk<kMask> walk(un);
      if (kMask && any_keys) next_mask = fetch_mask(walk.jt);

      for (bool first = true; walk.more(); first = false, ++n_s) {
        const int jt = walk.jt;
        const uint32_t mask_bits = next_mask;
        walk.next();
        if (kMask && walk.more()) next_mask = fetch_mask(walk.jt);
        ok = mbar_wait_warp(bar_s_full(t), n_s & 1, limit);
        if (!ok) break;
        tc_fence_after();
        bool whole = (jt + 1) * 128 <= lim_all;            // all 128 keys count for all rows of the tile
        uint32_t bits[4] = {~0u, ~0u, ~0u, ~0u};           // the mask's word on them
        if (kMask) {
#pragma unroll
          for (int e = 0; e < 4; ++e) bits[e] = __ballot_sync(0xffffffffu, (mask_bits >> e) & 1u);
          whole = whole && (bits[0] & bits[1] & bits[2] & bits[3]) == ~0u;
        }
        // In two halves: the second half of S is still on its way while the first is exponentiated, and the first half of P is on
        // its way to tensor memory while the second is.  (Also fewer registers: 128 scores and 32 packed pairs at a time.)  The common
        // case has a copy of its own, and so has the redo: with one copy for all the kernel took 5 % longer, as a loop 30 %.
        uint32_t r[128];
        uint32_t (&r_lo)[64] = *reinterpret_cast<uint32_t(*)[64]>(&r[0]);
        uint32_t (&r_hi)[64] = *reinterpret_cast<uint32_t(*)[64]>(&r[64]);
        uint32_t pk[32];
        tmem_ld32(tS, *reinterpret_cast<uint32_t(*)[32]>(&r[0]));
        tmem_ld32(tS + 32, *reinterpret_cast<uint32_t(*)[32]>(&r[32]));
        tmem_wait_ld_dep64(r_lo);
        tmem_ld32(tS + 64, *reinterpret_cast<uint32_t(*)[32]>(&r[64]));
        tmem_ld32(tS + 96, *reinterpret_cast<uint32_t(*)[32]>(&r[96]));
        float acc[4];
        if (whole && started) {
          const float mc = m_ref * c;
          acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
          softmax_half(r_lo, c, mc, pk, acc);
          tmem_wait_ld_dep64(r_hi);
          tmem_st32(tS, pk);
          softmax_half(r_hi, c, mc, pk, acc);
          seen = true;
        } else {
          tmem_wait_ld_dep64(r_hi);
          if (!whole) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t valid = below(lim, jt * 128 + e * 32) & bits[e];
              seen = seen || valid != 0;
#pragma unroll
              for (int cc = 0; cc < 32; ++cc)
                if (((valid >> cc) & 1u) == 0) r[e * 32 + cc] = __float_as_uint(-CUDART_INF_F);
            }
          }
          // a row takes its reference from its first tile with a valid key; before that every term is 2^-inf
          if (m_ref == -CUDART_INF_F) m_ref = row_max128(r);
          started = __all_sync(0xffffffffu, !mine || m_ref != -CUDART_INF_F);
          seen = seen || whole;
          const float mc = m_ref == -CUDART_INF_F ? 0.f : m_ref * c;
          acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
          softmax_half(r_lo, c, mc, pk, acc);
          tmem_st32(tS, pk);
          softmax_half(r_hi, c, mc, pk, acc);
        }
        // No row maximum was taken.  All terms are positive, so a sum <= 2^8 proves that every term is; otherwise, if the maximum
        // has grown by more than 2^8, the reference moves and the tile is redone before its P is released.
        if (__any_sync(0xffffffffu, mine && !((acc[0] + acc[1]) + (acc[2] + acc[3]) <= 256.0f))) {
          const float mx = row_max128(r);
          const bool grow = mine && (mx - m_ref) * c > 8.0f;
          if (__any_sync(0xffffffffu, grow)) {
            if (lane == 0) atomicAdd(p.rescales, 1u);
            const float f = grow ? ex2_approx((m_ref - mx) * c) : 1.0f;
            if (grow) m_ref = mx;
            l *= f;
            if (!first) {
              ok = mbar_wait_warp(bar_o_done(t), (n_s - 1) & 1, limit);
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int cch = 0; cch < D / 16; ++cch) {
                uint32_t o[16];
                tmem_ld16(tO + cch * 16, o);
                tmem_wait_ld();
#pragma unroll
                for (int cc = 0; cc < 16; ++cc) o[cc] = __float_as_uint(__uint_as_float(o[cc]) * f);
                tmem_st16(tO + cch * 16, o);
              }
            }
            tmem_wait_st();                                // the stale P lands before its replacement
            const float mc = m_ref == -CUDART_INF_F ? 0.f : m_ref * c;
            acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
            softmax_half(r_lo, c, mc, pk, acc);
            tmem_st32(tS, pk);
            softmax_half(r_hi, c, mc, pk, acc);
          }
        }
        tmem_st32(tS + 32, pk);
        l += (acc[0] + acc[1]) + (acc[2] + acc[3]);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p_full(t));
      }
      if (!ok) break;

      // ---- epilogue
      if (any_keys) {
        ok = mbar_wait_warp(bar_o_done(t), (n_s - 1) & 1, limit);
        if (!ok) break;
        tc_fence_after();
      }
      if (un.part >= 0) {
        float* dst = p.partial + (un.part * 2 * tile_rows + t * tile_rows + row) * (D + 4);
#pragma unroll 1
        for (int cch = 0; cch < D / 32; ++cch) {
          uint32_t o[32];                                  // (without a valid key: whatever is there, and not used)
          tmem_ld32(tO + cch * 32, o);
          tmem_wait_ld();
          if (mine) {
#pragma unroll
            for (int cc = 0; cc < 32; cc += 4) *reinterpret_cast<uint4*>(dst + cch * 32 + cc) = make_uint4(o[cc], o[cc + 1], o[cc + 2], o[cc + 3]);
          }
        }
        if (mine) *reinterpret_cast<float4*>(dst + D) = make_float4(m_ref, l, seen ? 1.f : 0.f, 0.f);
      } else {
        // Rows are staged 64 columns at a time (16-byte chunks XOR-swizzled by row) and written by one box (kBoxes) where a warp's rows
        // are whole tokens of the sequence, otherwise with eight lanes per row, four rows at a time; a lane's eight places are found first, so
        // that its stores follow one another.  (25,216 rows x 40 heads over 512 states: 284 us with lanes' stores, 272 with boxes.)
        const float inv = 1.0f / l;
        uint8_t* stage = smem + L::kOffStage + warp * 4096;
        int own = lane;
        asm volatile("" : "+r"(own));                      // keeps what follows from it out of the registers of the main loop
        const int first_tok = un.t0 + t * p.tok_per_tile, left = un.n_tok - first_tok, ch = own & 7;
        __nv_bfloat16* base = p.a.out + (un.tok0 + first_tok) * p.a.o_tok + (long long)(un.kv_head * group) * p.a.o_head + ch * 8;
        const int warp_tok = (int)(wq * 32 * p.inv_group >> 16);           // where a warp's rows are whole tokens: its first
        const bool boxed = kBoxes && warp_tok + (int)(32 * p.inv_group >> 16) <= left;
        __nv_bfloat16* place[8];
        if (!boxed) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int tile_row = wq * 32 + 4 * e + (own >> 3);
            const int in_tile = (int)(tile_row * p.inv_group >> 16);       // token of the tile
            place[e] = tile_row < tile_rows && in_tile < left ? base + in_tile * p.a.o_tok + (tile_row - in_tile * group) * p.a.o_head : nullptr;
          }
        }
        const uint64_t pol_once = l2_policy_evict_first();
#pragma unroll 1
        for (int hf = 0; hf < L::kHalves; ++hf) {
          uint32_t o[64];                                  // (without key tiles: whatever is there, and not used)
          tmem_ld32(tO + hf * 64, *reinterpret_cast<uint32_t(*)[32]>(&o[0]));
          tmem_ld32(tO + hf * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&o[32]));
          tmem_wait_ld_dep64(o);
          if (kBoxes && lane == 0) bulk_wait_read_all();      // the last box has left the staging rows
          __syncwarp();
#pragma unroll
          for (int v = 0; v < 8; ++v) {
            uint4 w = make_uint4(0u, 0u, 0u, 0u);          // a row without a valid key is zeros
            if (seen) {
              w.x = pack_bf16x2(__uint_as_float(o[8 * v + 0]) * inv, __uint_as_float(o[8 * v + 1]) * inv);
              w.y = pack_bf16x2(__uint_as_float(o[8 * v + 2]) * inv, __uint_as_float(o[8 * v + 3]) * inv);
              w.z = pack_bf16x2(__uint_as_float(o[8 * v + 4]) * inv, __uint_as_float(o[8 * v + 5]) * inv);
              w.w = pack_bf16x2(__uint_as_float(o[8 * v + 6]) * inv, __uint_as_float(o[8 * v + 7]) * inv);
            }
            *reinterpret_cast<uint4*>(stage + own * 128 + ((v ^ ch) << 4)) = w;
          }
          if (boxed) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store_3d_hint(&tm_o, sbase + L::kOffStage + warp * 4096, hf * 64, un.kv_head * group, (int)un.tok0 + first_tok + warp_tok, pol_once);
              bulk_commit_group();
            }
            continue;
          }
          __syncwarp();
          uint4 w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int rr = 4 * e + (own >> 3);
            w[e] = *reinterpret_cast<const uint4*>(stage + rr * 128 + ((ch ^ (rr & 7)) << 4));
          }
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (place[e] != nullptr) st_global_evict_first(place[e] + hf * 64, w[e], pol_once);
        }
      }
      release_unit(u);
    }
    if (kBoxes && lane == 0) bulk_wait_all();
    if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutSoftmax);
  } else {
    setmaxnreg_dec<SOL_REGS_OTHER>();
  }

  if (warp == 8) {
    // =========================================================== loads
    const uint64_t pol_once = l2_policy_evict_first();
    const uint32_t q_bytes = (uint32_t)(p.tok_per_tile * p.a.group * 128 * L::kHalves);
    uint32_t it = 0, n_q[2] = {0, 0};
    bool ok = true;
    for (uint32_t u = 0;; ++u) {
      if (!wait_long(bar_u_full(u), round_of(u))) { ok = false; break; }
      const UnitDev& un = units[u & (kUnitRing - 1)];
      if (un.last) break;
      const int kv_head = un.kv_head, n = un.span.cap;
      const int* table = un.span.table;
      const long long begin = un.span.begin;
      if (un.n_keys > 0) {
        for (int t = 0; t < un.n_tiles && ok; ++t) {
          ok = mbar_wait_warp(bar_q_empty(t), (n_q[t] & 1) ^ 1u, limit);
          if (!ok) break;
          ++n_q[t];
          if (lane == 0) {
            mbar_arrive_expect_tx(bar_q_full(t), q_bytes);
#pragma unroll
            for (int hf = 0; hf < L::kHalves; ++hf)
              tma_load_3d_hint(sQ + t * L::kTile + hf * L::kHalfBytes, &tm_q, bar_q_full(t), hf * 64, kv_head * p.a.group,
                               (int)un.tok0 + un.t0 + t * p.tok_per_tile, pol_once);
          }
          __syncwarp();
        }
        // a lane's page of a key tile; tokens beyond the keys, and entries that name no page, load zeros (a coordinate past the end)
        auto page_of = [&](int jt) {
          const int key = jt * 128 + lane * p.box_rows;
          if (lane * p.box_rows >= 128 || key >= n) return (int)p.d.c.n_pages;
          const int page = table[key / p.d.c.page];
          return page >= 0 && page < p.d.c.n_pages ? page : (int)p.d.c.n_pages;
        };
        int next_page = 0;
        TileWalk<kMask> walk(un);
        if (kPaged && ok) next_page = page_of(walk.jt);
        bool near = false;
        while (walk.more() && ok) {
          const int jt = walk.jt;
          walk.next();
          if (!near && walk.left <= kNear) {
            near = true;
            if (lane == 0) mbar_arrive(bar_near(u));
          }
          const int page = next_page;
          if (kPaged && walk.more()) next_page = page_of(walk.jt);
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const uint32_t stage = it % L::kStages;
            ok = mbar_wait_warp(bar_kv_empty(stage), ((it / L::kStages) & 1) ^ 1u, limit);
            if (!ok) break;
            const uint32_t dst = sKV + stage * L::kTile;
            const CUtensorMap* tm = kv ? &tm_v : &tm_k;
            if (lane == 0) mbar_arrive_expect_tx(bar_kv_full(stage), L::kTile);
            __syncwarp();
            if (kPaged) {
              if (lane * p.box_rows < 128) {
                const int in_page = (jt * 128 + lane * p.box_rows) % p.d.c.page;
#pragma unroll
                for (int hf = 0; hf < L::kHalves; ++hf)
                  tma_load_4d(dst + hf * L::kHalfBytes + lane * p.box_rows * 128, tm, bar_kv_full(stage), hf * 64, kv_head, in_page, page);
              }
            } else if (lane == 0) {
#pragma unroll
              for (int hf = 0; hf < L::kHalves; ++hf)
                tma_load_3d(dst + hf * L::kHalfBytes, tm, bar_kv_full(stage), hf * 64, kv_head, (int)(begin + jt * 128));
            }
            __syncwarp();
            ++it;
          }
        }
      } else if (lane == 0) {
        mbar_arrive(bar_near(u));
      }
      if (!ok) break;
      release_unit(u);
    }
    if (!ok) {
      if (lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutProducer);
      // copies in flight land before the shared memory is given back
      for (int t = 0; t < 2; ++t)
        if (n_q[t] > 0) mbar_wait_warp(bar_q_full(t), (n_q[t] - 1) & 1, limit);
      const uint32_t first = it > (uint32_t)L::kStages ? it - L::kStages : 0u;
      for (uint32_t j = first; j < it; ++j) mbar_wait_warp(bar_kv_full(j % L::kStages), (j / L::kStages) & 1u, limit);
    }
  } else if (warp == 9) {
    // =========================================================== MMA issuer (the warp runs convergently, one elected lane issues)
    constexpr uint32_t idesc_qk = idesc_bf16_f32(128, 128, false);
    constexpr uint32_t idesc_pv = idesc_bf16_f32(128, D, true);
    const uint32_t hi_k = smem_desc_hi_sw128(1024), hi_v = smem_desc_hi_sw128(p.v_sbo);
    const uint32_t q_lo0 = smem_desc_lo(sQ, 16), q_lo1 = smem_desc_lo(sQ + L::kTile, 16);
    const uint32_t k_lo_base = smem_desc_lo(sKV, 16), v_lo_base = smem_desc_lo(sKV, p.v_lbo);
    constexpr uint32_t kStageStep = L::kTile >> 4;
    const uint32_t tS0 = tmem_base, tS1 = tmem_base + 128, tO0 = tmem_base + 256, tO1 = tmem_base + 256 + D;
    auto issue_qk = [&](uint32_t d_tmem, uint32_t q_lo, uint32_t stage) {
      const uint32_t k_lo = k_lo_base + stage * kStageStep;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t off = ((k >> 2) * L::kHalfBytes + (k & 3) * 32) >> 4;
        if (k == 0) mma_ss_elect<false>(d_tmem, q_lo + off, k_lo + off, hi_k, idesc_qk, 0u);
        else        mma_ss_elect<true>(d_tmem, q_lo + off, k_lo + off, hi_k, idesc_qk, 1u);
      }
    };
    auto issue_pv = [&](uint32_t d_tmem, uint32_t p_tmem, uint32_t stage, bool acc) {
      const uint32_t v_lo = v_lo_base + stage * kStageStep;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k == 0) mma_ts_elect<false>(d_tmem, p_tmem, v_lo, hi_v, idesc_pv, acc ? 1u : 0u);
        else        mma_ts_elect<true>(d_tmem, p_tmem + k * 8, v_lo + k * (2048 >> 4), hi_v, idesc_pv, 1u);
      }
    };
    uint32_t it = 0, n_v = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (!mbar_wait_warp(bar, parity, limit)) { ok = false; return false; }
      tc_fence_after();
      return true;
    };
    auto stage_of = [&](uint32_t n) { return n % L::kStages; };
    auto full = [&](uint32_t n) { return wait(bar_kv_full(n % L::kStages), (n / L::kStages) & 1); };
    // The next unit: kNone, kEmpty (it has no key tiles, the softmax warps see to its rows) or kTiles.
    enum { kNone, kEmpty, kTiles };
    uint32_t u = 0;
    int n_proc = 0;
    bool two = false, withhold = false;
    auto draw = [&]() {
      if (!wait_long(bar_u_full(u), round_of(u))) { ok = false; return (int)kNone; }
      const UnitDev& un = units[u & (kUnitRing - 1)];
      if (un.last) return (int)kNone;
      n_proc = un.n_keys;
      two = un.n_tiles == 2;
      withhold = un.withhold != 0;
      release_unit(u++);
      return (int)(n_proc > 0 ? kTiles : kEmpty);
    };
    // One stream of key tiles through units that follow one another: scores of tile 0 for the next key tile, which may be the next
    // unit's first, follow the product of this one, so that a unit's end looks to the tensor core like its middle.  (An empty unit
    // ends the stream: looking past it could wait for this unit's own end.)
    while (ok) {
      int what = draw();
      while (what == kEmpty) what = draw();
      if (what != kTiles) break;
      // (withhold, a test hook: a signal is left out, so that the waits downstream run into their limit)
      {
        const uint32_t k_st = stage_of(it);
        if (!wait(bar_q_full(0), n_q[0] & 1) || !full(it)) break;
        ++n_q[0];
        issue_qk(tS0, q_lo0, k_st);
        if (two || !withhold) tc_commit_elect(bar_s_full(0));
        if (n_proc == 1) tc_commit_elect(bar_q_empty(0));
        if (two) {
          if (!wait(bar_q_full(1), n_q[1] & 1)) break;
          ++n_q[1];
          issue_qk(tS1, q_lo1, k_st);
          if (!withhold) tc_commit_elect(bar_s_full(1));
          if (n_proc == 1) tc_commit_elect(bar_q_empty(1));
        }
        tc_commit_elect(bar_kv_empty(k_st));
      }
      bool have = true;
      int i = 0;
      while (have && ok) {
        const uint32_t v_it = it + 1, next = it + 2;
        const bool now_two = two, first = i == 0;
        it += 2;
        if (!full(v_it) || !wait(bar_v_clean(n_v), (n_v / L::kVRing) & 1)) break;
        ++n_v;
        if (!wait(bar_p_full(0), n_p[0] & 1)) break;
        ++n_p[0];
        issue_pv(tO0, tS0, stage_of(v_it), !first);
        tc_commit_elect(bar_o_done(0));
        bool fresh = false;                                  // the next key tile is the first of another unit
        if (++i == n_proc) {
          what = draw();
          if (!ok) break;
          have = what == kTiles;
          fresh = true;
          i = 0;
        }
        if (have) {
          if (fresh) {
            if (!wait(bar_q_full(0), n_q[0] & 1)) break;
            ++n_q[0];
          }
          if (!full(next)) break;
          issue_qk(tS0, q_lo0, stage_of(next));
          tc_commit_elect(bar_s_full(0));
          if (i + 1 == n_proc) tc_commit_elect(bar_q_empty(0));
        }
        if (now_two) {
          if (!wait(bar_p_full(1), n_p[1] & 1)) break;
          ++n_p[1];
          issue_pv(tO1, tS1, stage_of(v_it), !first);
          tc_commit_elect(bar_o_done(1));
        }
        tc_commit_elect(bar_kv_empty(stage_of(v_it)));
        if (have) {
          if (two) {
            if (fresh) {
              if (!wait(bar_q_full(1), n_q[1] & 1)) break;
              ++n_q[1];
            }
            issue_qk(tS1, q_lo1, stage_of(next));
            tc_commit_elect(bar_s_full(1));
            if (i + 1 == n_proc) tc_commit_elect(bar_q_empty(1));
          }
          tc_commit_elect(bar_kv_empty(stage_of(next)));
        }
      }
      if (what == kNone) break;
    }
    if (!ok) {
      if (lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutMma);
      tc_commit_elect(bar_drain);                          // products in flight end before tensor memory is released
      mbar_wait_warp(bar_drain, 0, limit);
    }
  } else if (warp == 10) {
    // =========================================================== takes units
    bool ok = true;
    const int per_unit = 2 * p.tok_per_tile;
    int* order = reinterpret_cast<int*>(smem + L::kOffOrder);              // by rank, most keys first: sequence,
    unsigned int* start = reinterpret_cast<unsigned int*>(order) + kSortedSeqs;   // its first item,
    int* n_unit = order + 2 * kSortedSeqs;                                 // its units, all heads,
    int* n_part = order + 3 * kSortedSeqs;                                 // parts of each,
    int* part0 = order + 4 * kSortedSeqs;                                  // its first partial rows (where there are several)
    const bool sorted = p.a.n_seqs <= kSortedSeqs;
    SeqNote* notes = reinterpret_cast<SeqNote*>(smem + L::kOffSeqs);       // by place in the schedule
    int looked_at = -1;                                    // the sequence whose live key tiles these are
    uint32_t live = 0;
    // whole units, then `tail` units of `tail_split` parts (one kind of units, or more sequences than are sorted)
    long long n_whole = p.n_whole, tail = p.n_tail, n_items = p.n_whole + p.n_tail * p.n_split;
    int tail_split = p.n_split, joins = p.n_split > 1 ? (int)p.n_tail : 0;
    if (sorted) {
      int keys = -1, units = 0;
      if (lane < p.a.n_seqs) {
        const SeqDev& sq = p.a.seqs[lane];
        const Span sp = find_span<kPaged>(p.d, sq.seq_id);
        keys = sp.idle ? -1 : sp.n;
        notes[lane] = SeqNote{kPaged ? (p.d.streams != nullptr ? p.d.streams[sq.seq_id] : sq.seq_id) : (int)sp.begin, keys, sp.cap, (int)sq.tok_start, sq.n_tokens};
        units = sp.idle || sp.n == 0 ? 0 : (sq.n_tokens + per_unit - 1) / per_unit * p.d.c.kv_heads;
      }
      int rank = 0;
      for (int j = 0; j < p.a.n_seqs; ++j) {
        const int other = __shfl_sync(0xffffffffu, keys, j);
        rank += other > keys || (other == keys && j < lane) ? 1 : 0;
      }
      if (lane >= p.a.n_seqs) rank = lane;
      const int tiles = keys > 0 ? (keys + 127) >> 7 : 0;
      // How to split the keys: lane i weighs parts of 1 / (i + 1) of the longest sequence's key tiles.  The unit of cost is a key tile
      // (some 2 us); a part costs 2 for its start and end, its partial rows 0.03 on their way through memory, a join 1.5.  Units of
      // one kind are dealt in whole waves; a mixture, largest first, ends 0.15 of a part late and
      // has whole waves of its large parts.  (Four streams of 7 to 100 tiles: 342 us
      // unsplit, 377 us in thirds of the longest; 40 units of 147 tiles beside small ones: 372 and 150 us.)
      const int most = __shfl_sync(0xffffffffu, tiles, __ffs(__ballot_sync(0xffffffffu, rank == 0)) - 1);
      const int chunk = max(1, (most + lane) / (lane + 1));
      int flat = 0, items = 0, split_items = 0, large = 0;  // large: parts of more than half of the largest
      float work = 0.f, large_work = 0.f;
      bool one_kind = true;
      for (int j = 0; j < p.a.n_seqs; ++j) {
        const int t = __shfl_sync(0xffffffffu, tiles, j), n = __shfl_sync(0xffffffffu, units, j);
        const int parts = (t + chunk - 1) / chunk;
        flat += n;
        items += n * max(parts, 1);
        if (parts > 1) split_items += n * parts;
        const float w = (float)n * (float)(t + 2 * max(parts, 1));
        work += w;
        if (2 * t > chunk * max(parts, 1)) {
          large += n * max(parts, 1);
          large_work += w;
        }
        one_kind = one_kind && (n == 0 || t == most);
      }
      const float joining = split_items > 0 ? 1.5f + 0.03f * split_items : 0.f;
      float cost = one_kind ? (float)((items + kPlanSms - 1) / kPlanSms) * (chunk + 2) : fmaxf(fmaxf(work * (1.f / kPlanSms), (float)(chunk + 2)), large_work / max(large, 1) * (float)((large + kPlanSms - 1) / kPlanSms)) + 0.15f * (chunk + 2);
      cost += joining;
      if (split_items > p.max_parts || (lane > 0 && chunk < 4)) cost = CUDART_INF_F;
      // ... or, for units of one kind, whole ones in whole waves and the rest in i + 1 parts each
      const int waves = flat / kPlanSms, rest = flat - waves * kPlanSms, rest_chunk = (most + lane) / (lane + 1);
      float tail_cost = (float)waves * (most + 2) + (float)((rest * (lane + 1) + kPlanSms - 1) / kPlanSms) * (rest_chunk + 2) + 1.5f + 0.03f * rest * (lane + 1);
      if (!one_kind || waves == 0 || rest == 0 || lane == 0 || rest_chunk < 4 || rest * (lane + 1) > p.max_parts) tail_cost = CUDART_INF_F;
      int pick = tail_cost < cost ? lane + 32 : lane;
      float best = fminf(cost, tail_cost);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float c = __shfl_xor_sync(0xffffffffu, best, o);
        const int w = __shfl_xor_sync(0xffffffffu, pick, o);
        if (c < best || (c == best && w < pick)) { best = c; pick = w; }
      }
      const bool by_tail = pick >= 32;
      const int by_chunk = by_tail ? 0x7fffffff : __shfl_sync(0xffffffffu, chunk, pick & 31);
      const int parts = by_tail || tiles == 0 ? 1 : (tiles - 1) / by_chunk + 1;
      // the items in rank order
      order[rank] = lane;
      n_unit[rank] = units;
      n_part[rank] = parts;
      __syncwarp();
      const int my_items = n_unit[lane] * n_part[lane], my_parts = n_part[lane] > 1 ? my_items : 0;
      int upto = my_items, parts_upto = my_parts, joins_upto = n_part[lane] > 1 ? n_unit[lane] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o), y = __shfl_up_sync(0xffffffffu, parts_upto, o), z = __shfl_up_sync(0xffffffffu, joins_upto, o);
        if (lane >= o) { upto += x; parts_upto += y; joins_upto += z; }
      }
      start[lane] = (unsigned int)(upto - my_items);
      part0[lane] = parts_upto - my_parts;
      __syncwarp();
      n_whole = __shfl_sync(0xffffffffu, upto, 31);
      joins = __shfl_sync(0xffffffffu, joins_upto, 31);
      tail = 0;
      tail_split = 1;
      n_items = n_whole;
      if (by_tail) {
        n_whole = (long long)waves * kPlanSms;
        tail = rest;
        tail_split = (pick & 31) + 1;
        n_items = n_whole + tail * tail_split;
        joins = rest;
      }
    }
    if (p.join_count != nullptr && blockIdx.x == 0 && lane == 0) *p.join_count = joins;
    bool drawn = false, behind_long = false;
    for (uint32_t u = 0;; ++u) {
      // Behind a long unit an item is drawn when the unit's last key tiles are being loaded, not sooner: it could wait there while other
      // CTAs have nothing left (four streams of 7 to 100 key tiles: 349 us drawn a unit ahead, a quarter of it idle).  Behind a short
      // one it is drawn at once: looking it up must not hold it back (packed cross attention: 162 and 149 us).
      if (behind_long && !wait_long(bar_near(u - 1), round_of(u - 1))) { ok = false; break; }
      if (u >= (uint32_t)kUnitRing && !wait_long(bar_u_empty(u), round_of(u) ^ 1u)) { ok = false; break; }
      int last = 0;
      for (;;) {
        // the first item of a CTA is its own number; the others come from the counter
        unsigned int at = blockIdx.x;
        if (drawn) {
          if (lane == 0) at = atomicAdd(p.counter, 1u);
          at = __shfl_sync(0xffffffffu, at, 0) + gridDim.x;
        }
        if (at >= n_items) {
          // every CTA draws one number past the items; the one that draws the last of them leaves the counter as it was found
          if (lane == 0) {
            const unsigned int draws = (n_items > gridDim.x ? (unsigned int)n_items - gridDim.x : 0u) + gridDim.x;
            const unsigned int mine = drawn ? at - gridDim.x : atomicAdd(p.counter, 1u);
            if (mine + 1 == draws) *p.counter = 0u;
          }
          last = 1;
          break;
        }
        drawn = true;
        const bool in_tail = at >= n_whole;
        const long long tail_unit = in_tail ? (at - n_whole) % tail : 0;
        const long long flat = in_tail ? n_whole + tail_unit : at;
        int split = in_tail ? (int)((at - n_whole) / tail) : 0, n_split = in_tail ? tail_split : 1;
        int first_part = (int)tail_unit * tail_split, join_at = (int)tail_unit;
        // ---- which sequence, K/V head and rows
        int si = 0, kv_head = 0;
        long long t0 = -1;
        if (sorted) {
          const int slot = 31 - __clz(__ballot_sync(0xffffffffu, start[lane] <= flat && lane < p.a.n_seqs));
          si = order[slot];
          const int n = (notes[si].n_tok + per_unit - 1) / per_unit;
          int local = (int)(flat - start[slot]);
          if (n_part[slot] > 1) {                          // part by part: units that run together share their keys
            n_split = n_part[slot];
            split = local / n_unit[slot];
            local -= split * n_unit[slot];
            first_part = part0[slot] + local * n_split;
            join_at = local;
            for (int r = 0; r < slot; ++r) join_at += n_part[r] > 1 ? n_unit[r] : 0;
          }
          kv_head = local / n;
          t0 = (long long)(local - kv_head * n) * per_unit;
        } else {
          long long first;
          kv_head = (int)(flat / p.units);
          si = find_sequence(p.a, flat % p.units, per_unit * p.a.group, &first);
          t0 = (flat % p.units - first) * per_unit;
          if (t0 >= p.a.seqs[si].n_tokens) t0 = -1;
        }
        UnitDev un{};
        un.t0 = (int)t0;
        un.kv_head = kv_head;
        if (sorted) {
          const SeqNote& q = notes[si];
          un.tok0 = q.tok0;
          un.n_tok = q.n_tok;
          un.span.n = q.n;
          un.span.cap = q.cap;
          un.span.begin = q.at;
          un.span.table = kPaged ? p.d.c.table + q.at * p.d.c.width : nullptr;
          un.span.mask = p.d.mask != nullptr ? p.d.mask + (kPaged ? q.at * p.d.mask_stride : (long long)q.at) : nullptr;
        } else if (t0 >= 0) {
          const SeqDev& sq = p.a.seqs[si];
          un.span = find_span<kPaged>(p.d, sq.seq_id);
          un.n_tok = sq.n_tokens;
          un.tok0 = sq.tok_start;
        }
        const bool none = t0 < 0 || un.span.idle;
        if (n_split > 1 && split == 0 && lane == 0) p.join[join_at] = JoinUnit{un.tok0, none ? 0 : un.t0, none ? 0 : un.n_tok, kv_head, first_part, n_split, 0};
        if (none) continue;
        un.part = n_split > 1 ? first_part + split : -1;
        un.n_tiles = un.n_tok - un.t0 > p.tok_per_tile ? 2 : 1;
        un.lim[0] = key_limit(un.span, un.n_tok, un.t0, p.a.causal);
        un.lim[1] = key_limit(un.span, un.n_tok, un.t0 + p.tok_per_tile, p.a.causal);
        const int most = key_limit(un.span, un.n_tok, min(un.n_tok, un.t0 + per_unit) - 1, p.a.causal);
        const int tiles = (most + 127) >> 7, per = (tiles + n_split - 1) / n_split;
        un.tile_begin = min(tiles, split * per);
        un.n_keys = min(tiles, un.tile_begin + per) - un.tile_begin;
        if (kMask && tiles <= 32) {
          // a tile without a valid key (the padding of a prompt, say) is left out; looked up once per sequence
          if (si != looked_at) {
            looked_at = si;
            live = 0;
            for (int jt = 0; jt * 128 < un.span.cap && jt < 32; jt += 4) {  // the loads of four tiles together
              bool on[4] = {false, false, false, false};
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int key = jt * 128 + e * 32 + lane;
                const bool counts = key < un.span.cap && un.span.mask[key] != 0;
                on[e >> 2] |= counts;
              }
#pragma unroll
              for (int e = 0; e < 4; ++e) live |= (__any_sync(0xffffffffu, on[e]) ? 1u : 0u) << (jt + e);
            }
          }
          const uint32_t mine = live & (un.n_keys > 0 ? (0xffffffffu >> (32 - un.n_keys)) << un.tile_begin : 0u);
          un.live = mine;
          un.n_keys = __popc(mine);
        }
        un.withhold = p.fault_inject == 1u && at == 0;
        if (lane == 0) units[u & (kUnitRing - 1)] = un;
        behind_long = un.n_keys > kNear;
        break;
      }
      if (lane == 0) {
        if (last) units[u & (kUnitRing - 1)].last = 1;
        mbar_arrive(bar_u_full(u));
      }
      if (last) break;
    }
    if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutProducer);
  } else if (warp == 11) {
    // =========================================================== values of keys that do not count
    uint32_t it = 0, n_v = 0;
    bool ok = true;
    for (uint32_t u = 0; ok; ++u) {
      if (!wait_long(bar_u_full(u), round_of(u))) { ok = false; break; }
      const UnitDev& un = units[u & (kUnitRing - 1)];
      if (un.last) break;
      TileWalk<kMask> walk(un);
      const int cap = un.span.cap;
      const uint8_t* mask = kMask ? un.span.mask : nullptr;
      release_unit(u);
      for (; walk.more(); walk.next()) {
        const int jt = walk.jt;
        const uint32_t v_it = it + 1, stage = v_it % L::kStages;
        it += 2;
        uint32_t drop = 0;                                 // bit e: key 32 e + lane of the tile does not count
        if (kMask || (jt + 1) * 128 > cap) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = jt * 128 + e * 32 + lane;
            if (key >= cap || (kMask && mask[key] == 0)) drop |= 1u << e;
          }
        }
        if (!mbar_wait_warp(bar_kv_full(stage), (v_it / L::kStages) & 1, limit)) { ok = false; break; }
        if (__any_sync(0xffffffffu, drop != 0)) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((drop >> e) & 1u) {
              uint8_t* at = smem + L::kOffKV + stage * L::kTile + (e * 32 + lane) * 128;
#pragma unroll
              for (int hf = 0; hf < L::kHalves; ++hf)
#pragma unroll
                for (int ch = 0; ch < 8; ++ch)             // (lanes start at different chunks: different banks)
                  *reinterpret_cast<uint4*>(at + hf * L::kHalfBytes + (((ch + lane) & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
            }
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_v_clean(n_v));
        ++n_v;
      }
    }
    if (!ok && lane == 0) atomicCAS(p.status, 0u, kStatusTimeoutProducer);
  }

  // ---- everyone is done with tensor memory and shared memory before they are released
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

}  // namespace sol
