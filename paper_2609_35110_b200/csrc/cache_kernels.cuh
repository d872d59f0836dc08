// A K/V cache in pages: bringing new tokens in (norm, rotation, write), and opening, growing, thinning and closing streams.
//
// A cache is [layers][pages][page][kv_heads][head_dim]; token j of a stream is row j % page of page table[stream][j / page], in every
// layer.  refs[p] counts the streams that hold page p; a page is free while it is 0.  A page that several streams hold is full
// and never written again: forking shares full pages and copies the last, partly filled one at once.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "device_types.cuh"
#include "ptx_sm100.cuh"

namespace sol {

// One layer of a cache as the kernels that read or write tokens see it.
struct PagedDev {
  __nv_bfloat16* k;
  __nv_bfloat16* v;
  long long ks[3], vs[3];       // element strides {page, token, head}
  const int* table;
  const int* lens;
  long long width;              // columns of the table
  long long n_streams, n_pages;
  int page, kv_heads;
};

// Kernels of this family may be launched while their predecessor in the stream still runs (programmatic dependent launch): each waits
// for it here before it touches memory, and lets its own successor be launched at once, which saves some 3 us between short kernels.
// Such a kernel lives while its predecessor still writes, so what callers or predecessors write is read by plain loads: __ldg is for memory that
// nobody writes as long as the kernel lives (here: the plan's tables), and the compiler may move it across the wait.
__device__ __forceinline__ void chained_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void chained_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Tokens of a stream that the table has room for.
__device__ __forceinline__ long long stream_tokens(const PagedDev& c, long long stream) {
  const long long n = c.lens[stream], cap = c.width * c.page;
  return n < 0 ? 0 : n < cap ? n : cap;
}

// ---------------------------------------------------------------------------------------------
// New tokens of a plan's sequences into one layer of a cache: K and (optionally) Q are RMS-normalised per head, rotated by
// the token's (t, h, w), offset per sequence, and rounded once; V is copied.  Row i of a chunk of n tokens becomes token
// N - n + i of a stream of N.  Every value is read and written once, 45 us of HBM for 4,680 tokens x 40 heads x 128; it takes 66 us
// (0.288 GB, 4.4 TB/s): the barriers around a group's angles, the largest stall, and issuing instructions (63 % of the slots) bound it.
// 16 tokens x 40 / 8 heads: 6 us on the GPU.
//
// A block takes up to four neighbouring tokens at a time.  It finds their sequences and streams, and sends for the first rows of those that
// are not idle.  Then its threads find the angles of the tokens' pairs, one each, and the tokens' places in the cache: the angles from the
// plan's tables, or, where positions are offset, from position times frequency in fp64, brought to (-pi, pi] there (the tables end
// with the grid, and fp32 loses far positions).  Then a thread owns 16-byte chunks (8 dims) of rows, four rows at a time: the same head of
// the four tokens (kTokens = 4), or four heads of one (kTokens = 1: few tokens); all Q heads, then all K heads, then V.  A row's address
// is a base per token and an offset per head (found row by row they made 183 instructions per 8 values of a lane: 98 us; every thread
// finding its own angles: 106 us; one token at a time: 93 us).
// ---------------------------------------------------------------------------------------------
struct AppendArgs {
  const __nv_bfloat16* x[3];    // q, k, v of the new tokens (q may be nullptr)
  long long x_tok[3], x_head[3];
  __nv_bfloat16* q_out;         // dense [tokens][heads][D]
  const float* gain[2];         // of q and k, or nullptr
  float eps;
  const SeqDev* seqs;
  int n_seqs;
  long long total_tokens;
  const float2* tables;
  RopeGeom g;
  const int* streams;           // per sequence (caller's order), or nullptr: sequence s is stream s
  const int* pos0;              // [n_seqs][3] offsets of (t, h, w), or nullptr
  PagedDev c;
  const double* omega;          // frequency of pair j of head_dim / 2
};

template <int D, int kTokens>
__global__ void __launch_bounds__(256, 3) cache_append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kBatch = 4, kChunks = D / 8;
  __shared__ __align__(16) float2 angle[kTokens][D / 2];
  __shared__ __nv_bfloat16* place[3][kTokens];             // where a token's first Q, K and V head go; nullptr: nowhere
  __shared__ int found[kTokens], rotates[kTokens], home[kTokens];          // home: the token's stream, or -1: of an idle sequence
  const int rows_per_pass = blockDim.x / kChunks;
  const int chunk = threadIdx.x % kChunks, sub = threadIdx.x / kChunks;
  const unsigned lanes = __activemask();
  const int d1 = a.g.rope[0], d2 = d1 + a.g.rope[1], d3 = d2 + a.g.rope[2];
  const int turned = max(0, min(4, (d3 >> 1) - 4 * chunk));  // pairs of this thread's chunk that rotate; the rest pass as they are, infinities too
  // Step: a tensor and a batch of its heads.
  constexpr int kHeads = kBatch / kTokens;
  const int head_step = kHeads * rows_per_pass;
  const int q_steps = a.x[0] != nullptr ? (a.g.heads + head_step - 1) / head_step : 0, k_steps = (a.c.kv_heads + head_step - 1) / head_step;
  const int steps = q_steps + 2 * k_steps;
  auto step_of = [&](int it, int& which, int& n, int& h0) {
    which = it < q_steps ? 0 : it < q_steps + k_steps ? 1 : 2;
    n = which == 0 ? a.g.heads : a.c.kv_heads;
    h0 = (which == 0 ? it : which == 1 ? it - q_steps : it - q_steps - k_steps) * head_step + sub;
  };
  chained_wait();
  chained_next();

  for (long long tok0 = (long long)blockIdx.x * kTokens; tok0 < a.total_tokens; tok0 += (long long)gridDim.x * kTokens) {
    const int n_tok = (int)min((long long)kTokens, a.total_tokens - tok0);
    // ---- the tokens' sequences and streams; an idle sequence's rows are not read
    const int my_tok = threadIdx.x % kTokens;
    if (my_tok < n_tok)
      for (int s = threadIdx.x / kTokens; s < a.n_seqs; s += blockDim.x / kTokens) {
        const SeqDev& sq = a.seqs[s];
        if (tok0 + my_tok >= sq.tok_start && tok0 + my_tok < sq.tok_start + sq.n_tokens) {
          const long long stream = a.streams != nullptr ? a.streams[sq.seq_id] : sq.seq_id;
          found[my_tok] = s;
          home[my_tok] = stream >= 0 && stream < a.c.n_streams ? (int)stream : -1;
        }
      }
    __syncthreads();
    unsigned pick = 0;                                     // a byte per token: itself, or where it is not there or idle the first that is not
    int live = -1;
#pragma unroll
    for (int g = kTokens - 1; g >= 0; --g)
      if (g < n_tok && home[g] >= 0) live = g;
    if (live < 0) {
      __syncthreads();                                     // (homes have been read)
      continue;
    }
#pragma unroll
    for (int g = 0; g < kTokens; ++g) pick |= (unsigned)(g < n_tok && home[g] >= 0 ? g : live) << (8 * g);
    uint4 ahead[kBatch];
    auto load = [&](int it) {                              // (past the last head: that one again, not stored)
      int which, n, h0;
      step_of(it, which, n, h0);
      const long long x_tok = a.x_tok[which];
      const int x_head = (int)a.x_head[which];
      const __nv_bfloat16* src = a.x[which] + tok0 * x_tok + chunk * 8;
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int h = min(h0 + b / kTokens * rows_per_pass, n - 1);
        ahead[b] = *reinterpret_cast<const uint4*>(src + (int)((pick >> (8 * (b % kTokens))) & 255u) * x_tok + (long long)h * x_head);
      }
    };
    load(0);
    // ---- their angles and places
    for (int j = threadIdx.x; j < n_tok * (D / 2); j += blockDim.x) {
      const int g = j / (D / 2), pair = j % (D / 2);
      const SeqDev& sq = a.seqs[found[g]];
      const int local = (int)(tok0 + g - sq.tok_start), p = local - sq.text_len;
      const int d = 2 * pair;                              // first head dim of the pair
      float2 cs = make_float2(1.f, 0.f);
      if (p >= 0 && d < d3) {
        const int axis = d < d1 ? 0 : d < d2 ? 1 : 2;
        const int x = axis == 0 ? p / (sq.H * sq.W) : axis == 1 ? (p / sq.W) % sq.H : p % sq.W;
        if (a.pos0 != nullptr) {
          const double phi = (double)((long long)x + a.pos0[3 * sq.seq_id + axis]) * __ldg(a.omega + pair);
          const double turns = rint(phi * 0.15915494309189535);             // 1 / (2 pi)
          const double rest = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, phi));   // 2 pi in two parts
          sincosf((float)rest, &cs.y, &cs.x);
        } else {
          const int first = axis == 0 ? 0 : axis == 1 ? d1 : d2;
          cs = __ldg(&a.tables[a.g.tab_off[axis] + x * (a.g.rope[axis] >> 1) + ((d - first) >> 1)]);
        }
      }
      angle[g][pair] = cs;
    }
    if (threadIdx.x >= blockDim.x - 32) {                  // the last warp: places (the first ones may have more angles to find)
      const int lane = threadIdx.x & 31;
      for (int g = 0; g < n_tok; ++g) {
        const SeqDev& sq = a.seqs[found[g]];
        const long long stream = home[g];
        // Of several sequences with one stream the first counts: they would write the same rows.
        bool again = false;
        if (a.streams != nullptr)
          for (int s = lane; s < sq.seq_id; s += 32) again = again || a.streams[s] == stream;
        again = __any_sync(0xffffffffu, again);
        if (lane == 0) {
          place[0][g] = place[1][g] = place[2][g] = nullptr;
          if (stream >= 0) {                               // (otherwise an idle sequence)
            place[0][g] = a.q_out + (tok0 + g) * a.g.heads * (long long)D;
            const long long at = stream_tokens(a.c, stream) - sq.n_tokens + (tok0 + g - sq.tok_start);
            if (at >= 0 && !again) {
              const int page = a.c.table[stream * a.c.width + (int)at / a.c.page], row = (int)at % a.c.page;
              if (page >= 0 && page < a.c.n_pages) {       // (a table that names no page there: nothing is written)
                place[1][g] = a.c.k + page * a.c.ks[0] + row * a.c.ks[1];
                place[2][g] = a.c.v + page * a.c.vs[0] + row * a.c.vs[1];
              }
            }
          }
          rotates[g] = tok0 + g - sq.tok_start >= sq.text_len;
        }
      }
    }
    __syncthreads();

    // ---- the rows: Q, then K, with norm and rotation, then V as it is; the next step's loads are on their way during a step
#pragma unroll 1
    for (int it = 0; it < steps; ++it) {
      uint4 w[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) w[b] = ahead[b];
      if (it + 1 < steps) load(it + 1);
      int which, n, h0;
      step_of(it, which, n, h0);
      const int out_head = which == 0 ? D : which == 1 ? (int)a.c.ks[2] : (int)a.c.vs[2];
      float rinv[kBatch], gains[8];
      const bool norm = which < 2 && a.gain[which & 1] != nullptr;
      if (norm) {
          *reinterpret_cast<float4*>(&gains[0]) = *reinterpret_cast<const float4*>(a.gain[which & 1] + chunk * 8);
          *reinterpret_cast<float4*>(&gains[4]) = *(reinterpret_cast<const float4*>(a.gain[which & 1] + chunk * 8) + 1);
          // Sums of squares of the rows, by shuffles over a row's chunks; where they leave fp32's range, once more on scaled values.
          auto squares = [&](float scale, float (&ss)[kBatch]) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
              const uint32_t v[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
              ss[b] = 0.f;
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                float lo = __uint_as_float(v[u] << 16), hi = __uint_as_float(v[u] & 0xffff0000u);
                if (scale != 1.0f) { lo *= scale; hi *= scale; }
                ss[b] = fmaf(lo, lo, ss[b]);
                ss[b] = fmaf(hi, hi, ss[b]);
              }
            }
#pragma unroll
            for (int off = kChunks / 2; off > 0; off >>= 1)
#pragma unroll
              for (int b = 0; b < kBatch; ++b) ss[b] += __shfl_xor_sync(lanes, ss[b], off);
          };
          float ss[kBatch];
          squares(1.0f, ss);
          bool odd = false;
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            rinv[b] = rsqrtf(fmaf(ss[b], 1.0f / D, a.eps));
            odd = odd || !(ss[b] < 1e37f) || ss[b] < 1e-25f;
          }
          if (__any_sync(lanes, odd)) {
            float big[kBatch], tiny[kBatch];
            squares(0x1p-70f, big);
            squares(0x1p60f, tiny);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {             // (eps is nothing beside squares of 1e37 / D)
              if (!(ss[b] < 1e37f)) rinv[b] = rsqrtf(big[b] * (1.0f / D) + a.eps * 0x1p-120f * 0x1p-20f) * 0x1p-70f;
              else if (ss[b] < 1e-25f && a.eps < 1e-20f) rinv[b] = rsqrtf(tiny[b] * (1.0f / D) + a.eps * 0x1p120f) * 0x1p60f;
            }
          }
        }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int h = h0 + b / kTokens * rows_per_pass;
        __nv_bfloat16* dst = place[which][b % kTokens];
        if (h >= n || b % kTokens >= n_tok || dst == nullptr) continue;
        uint4 y = w[b];
        if (which < 2) {
          const uint32_t v[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
          float f[8];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            f[2 * u] = __uint_as_float(v[u] << 16);
            f[2 * u + 1] = __uint_as_float(v[u] & 0xffff0000u);
          }
          if (norm) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= rinv[b] * gains[e];
          }
          if (rotates[b % kTokens] != 0 && turned > 0) {
            const float4* cs = reinterpret_cast<const float4*>(&angle[b % kTokens][chunk * 4]);
#pragma unroll
            for (int u = 0; u < 2; ++u) {                  // two pairs: cos, sin, cos, sin
              const float4 t = cs[u];
              const float e0 = f[4 * u], o0 = f[4 * u + 1], e1 = f[4 * u + 2], o1 = f[4 * u + 3];
              if (2 * u < turned) {
                f[4 * u] = fmaf(e0, t.x, -(o0 * t.y));
                f[4 * u + 1] = fmaf(e0, t.y, o0 * t.x);
              }
              if (2 * u + 1 < turned) {
                f[4 * u + 2] = fmaf(e1, t.z, -(o1 * t.w));
                f[4 * u + 3] = fmaf(e1, t.w, o1 * t.z);
              }
            }
          }
          y = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        }
        *reinterpret_cast<uint4*>(dst + (long long)h * out_head + chunk * 8) = y;
      }
    }
    __syncthreads();                                       // places and angles are found anew for the next tokens
  }
}

// ---------------------------------------------------------------------------------------------
// Bookkeeping of streams and pages.  Requests of one call are served in their order: those that are in order take the free
// pages of the lowest index one after another, and a request that would need more than are left gets none.  Everything is
// integer arithmetic whose result does not depend on the order in which threads run.  One block: a call has tens of requests and
// thousands of pages, and what it costs is its launch and a chain of barriers (fork of 12 streams with its copies and two
// reservations, 34 us a set called one after another, 20 us replayed from a graph).
// ---------------------------------------------------------------------------------------------
enum : int { kCacheOk = 0, kCacheBadStream = 1, kCacheNoRoom = 2, kCacheNoPages = 3, kCacheNotEmpty = 4 };
constexpr int kMaxRequests = 2048;
constexpr int kBookThreads = 512, kKeepThreads = 1024;

struct BookArgs {
  int* table;
  int* lens;
  int* refs;
  long long width, n_streams, n_pages;
  int page;
  int n;                        // requests
  const int* streams;           // whose streams they name (fork: the new ones)
  const int* parents;           // fork only
  const int* amount;            // reserve only: tokens to add
  int* status;                  // [n], or nullptr
  // what the copying kernel is told (fork, compact)
  int2* moves;                  // [n][moves_cap] (source row, destination row) of the whole pool, rows counted over pages
  long long moves_cap;
  long long* moved;             // [n + 1] moves before request i
  // compact
  const uint8_t* keep;          // [n][keep_stride]
  long long keep_stride;
  int* kept;                    // [n] tokens that stay, or -1: the request is not in order
  int* first;                   // [n] the first dropped token (the length, if none)
  int* old_pages;               // [n][width] the table rows before the call
};

__device__ __forceinline__ int pages_of(int tokens, int page) { return tokens / page + (tokens % page != 0 ? 1 : 0); }
// The tokens a stream holds, within what its table row can hold.
__device__ __forceinline__ int stream_length(const BookArgs& a, long long stream) {
  const long long n = a.lens[stream], cap = a.width * a.page;
  return (int)(n < 0 ? 0 : n < cap ? n : cap);
}
// Sums over the block's threads, inclusive; `warp_sum` has 32 entries.  All threads call it; two barriers.
template <typename T>
__device__ __forceinline__ T block_scan(T x, long long* warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                                         // (the last call's sums have been read)
  if (lane == 31) warp_sum[warp] = x;
  __syncthreads();
  T t = lane < warp && lane < warps ? (T)warp_sum[lane] : (T)0;            // every warp sums the warps before it
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  return x + t;
}

struct BookSmem {
  long long warp_sum[32];
  int streams[kMaxRequests];     // as named
  int need[kMaxRequests];        // pages, or -1: refused
  int ends[kMaxRequests];        // need of the requests up to and including i (2^30 for all above that); later, rows to copy
  int extra[kMaxRequests];       // per request, as the kernel uses it
};

__device__ __forceinline__ void load_streams(const BookArgs& a, BookSmem& sm) {
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) sm.streams[i] = a.streams[i];
  __syncthreads();
}
// Is the stream of request i there, and not named by an earlier request?
__device__ __forceinline__ bool named_first(const BookArgs& a, const BookSmem& sm, int i) {
  const int s = sm.streams[i];
  if (s < 0 || s >= a.n_streams) return false;
  for (int j = 0; j < i; ++j)
    if (sm.streams[j] == s) return false;
  return true;
}

// Running sums of `of(i)` over the requests, into ends[]; returns the whole.  (Requests may ask for far more than there is.)
template <typename Of>
__device__ __forceinline__ int sum_up(const BookArgs& a, BookSmem& sm, const Of& of) {
  int before = 0;
  for (int i0 = 0; i0 < a.n; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    const long long s = before + block_scan<long long>(i < a.n ? of(i) : 0, sm.warp_sum);
    if (i < a.n) sm.ends[i] = (int)min(s, 1ll << 30);
    __syncthreads();
    before = sm.ends[min(i0 + (int)blockDim.x, a.n) - 1];
  }
  return before;
}

// Walks over the free pages, lowest index first, until `wanted` have been seen: take(rank, page).  Returns how many there were.
template <typename Take>
__device__ __forceinline__ int walk_free(const BookArgs& a, BookSmem& sm, int wanted, const Take& take) {
  constexpr int kEach = 8;                                 // neighbouring pages per thread and turn
  int found = 0;
  for (long long p0 = 0; p0 < a.n_pages && found < wanted; p0 += kEach * blockDim.x) {
    const long long first = p0 + kEach * threadIdx.x;
    unsigned bits = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (first + e < a.n_pages && a.refs[first + e] == 0) bits |= 1u << e;
    const int mine = __popc(bits), upto = block_scan<int>(mine, sm.warp_sum);
    int rank = found + upto - mine;
    for (; bits != 0; bits &= bits - 1, ++rank)
      if (rank < wanted) take(rank, (int)(first + __ffs(bits) - 1));
    if (threadIdx.x == blockDim.x - 1) sm.warp_sum[31] = upto;             // (read by no scan: there are fewer than 32 warps)
    __syncthreads();
    found += (int)sm.warp_sum[31];
  }
  return min(found, wanted);
}
static_assert(kBookThreads / 32 < 32, "walk_free keeps a sum in the last entry");

// Pages for requests with need[i] > 0, in their order: served(i) tells which get theirs, give(i, k, page) hands request i its k-th.
// The free pages are counted first, so that a request that cannot be served takes none.
struct Served {
  int there;
  __device__ __forceinline__ bool operator()(const BookSmem& sm, int i) const { return sm.need[i] >= 0 && !(sm.need[i] > 0 && sm.ends[i] > there); }
};
template <typename Give>
__device__ __forceinline__ Served allocate(const BookArgs& a, BookSmem& sm, const Give& give) {
  __syncthreads();
  const int wanted = sum_up(a, sm, [&](int i) { return max(sm.need[i], 0); });
  const Served served{walk_free(a, sm, wanted, [](int, int) {})};
  for (int i = threadIdx.x; i < a.n; i += blockDim.x)
    if (sm.need[i] > 0 && !served(sm, i) && a.status != nullptr) a.status[i] = kCacheNoPages;
  __syncthreads();
  walk_free(a, sm, served.there, [&](int rank, int p) {
    int lo = 0, hi = a.n - 1;                                              // the first request whose running sum exceeds the rank
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (sm.ends[mid] > rank) hi = mid; else lo = mid + 1;
    }
    if (sm.ends[lo] > served.there) return;
    give(lo, rank - (sm.ends[lo] - sm.need[lo]), p);
    a.refs[p] = 1;
  });
  __syncthreads();
  return served;
}

// Closing streams: their pages lose a holder.
__global__ void __launch_bounds__(kBookThreads) cache_free_kernel(const BookArgs a) {
  extern __shared__ __align__(16) unsigned char book_raw[];
  BookSmem& sm = *reinterpret_cast<BookSmem*>(book_raw);
  chained_wait();
  chained_next();
  load_streams(a, sm);
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < a.n; i += blockDim.x >> 5) {          // a warp per request
    bool ok = false;
    if (lane == 0) {
      ok = named_first(a, sm, i);
      if (a.status != nullptr) a.status[i] = ok ? kCacheOk : kCacheBadStream;
    }
    if (!__any_sync(0xffffffffu, ok)) continue;
    const long long s = sm.streams[i];
    const int held = pages_of(stream_length(a, s), a.page);
    for (int c = lane; c < held; c += 32) {
      const int p = a.table[s * a.width + c];
      if (p >= 0 && p < a.n_pages) atomicSub(a.refs + p, 1);
      a.table[s * a.width + c] = -1;
    }
    __syncwarp();
    if (lane == 0) a.lens[s] = 0;
  }
}

// Growing streams: pages for `amount` more tokens, and the length with them.
__global__ void __launch_bounds__(kBookThreads) cache_reserve_kernel(const BookArgs a) {
  extern __shared__ __align__(16) unsigned char book_raw[];
  BookSmem& sm = *reinterpret_cast<BookSmem*>(book_raw);
  chained_wait();
  chained_next();
  load_streams(a, sm);
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    int need = -1, st = kCacheBadStream;
    if (named_first(a, sm, i) && a.amount[i] >= 0) {
      const int len = stream_length(a, sm.streams[i]);
      const long long want = (long long)len + a.amount[i];
      sm.extra[i] = pages_of(len, a.page);
      st = kCacheNoRoom;
      if (want <= a.width * a.page && want <= 0x7fffffffll) {
        st = kCacheOk;
        need = pages_of((int)want, a.page) - sm.extra[i];
      }
    }
    sm.need[i] = need;
    if (a.status != nullptr) a.status[i] = st;
  }
  const Served served = allocate(a, sm, [&](int i, int k, int p) { a.table[sm.streams[i] * a.width + sm.extra[i] + k] = p; });
  for (int i = threadIdx.x; i < a.n; i += blockDim.x)
    if (served(sm, i)) a.lens[sm.streams[i]] = stream_length(a, sm.streams[i]) + a.amount[i];
}

// Opening streams as branches of others: full pages are shared, the last, partly filled one is copied (by cache_move_kernel).
__global__ void __launch_bounds__(kBookThreads) cache_fork_kernel(const BookArgs a) {
  extern __shared__ __align__(16) unsigned char book_raw[];
  BookSmem& sm = *reinterpret_cast<BookSmem*>(book_raw);
  int* len = sm.extra;                                     // of the parents, before anything changes
  chained_wait();
  chained_next();
  load_streams(a, sm);
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    int st = kCacheBadStream, need = -1;
    const int parent = a.parents[i];
    len[i] = 0;
    if (parent >= 0 && parent < a.n_streams && named_first(a, sm, i)) {
      st = kCacheNotEmpty;
      const int old = stream_length(a, parent);
      if (stream_length(a, sm.streams[i]) == 0) {
        st = kCacheOk;
        len[i] = old;
        need = old % a.page != 0 ? 1 : 0;
      }
    }
    sm.need[i] = need;
    if (a.status != nullptr) a.status[i] = st;
  }
  const Served served = allocate(a, sm, [&](int i, int, int p) { a.table[sm.streams[i] * a.width + len[i] / a.page] = p; });
  // one warp per request: the shared pages, and which rows of the last one have to be copied
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < a.n; i += blockDim.x >> 5) {
    if (!served(sm, i)) continue;
    const long long s = sm.streams[i], parent = a.parents[i];
    const int full = len[i] / a.page, rest = len[i] % a.page;
    for (int c = lane; c < full; c += 32) {
      const int p = a.table[parent * a.width + c];
      a.table[s * a.width + c] = p;
      if (p >= 0 && p < a.n_pages) atomicAdd(a.refs + p, 1);
    }
    if (rest > 0) {
      const int from = a.table[parent * a.width + full], to = a.table[s * a.width + full];
      const bool there_is = from >= 0 && from < a.n_pages;
      for (int r = lane; r < rest; r += 32)
        a.moves[i * a.moves_cap + r] = make_int2(there_is ? from * a.page + r : -1, to * a.page + r);
    }
    __syncwarp();
    if (lane == 0) a.lens[s] = len[i];
  }
  __syncthreads();
  // rows to copy before request i
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) sm.need[i] = sm.need[i] > 0 && served(sm, i) ? len[i] % a.page : 0;
  __syncthreads();
  sum_up(a, sm, [&](int i) { return sm.need[i]; });
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) a.moved[i + 1] = sm.ends[i];
  if (threadIdx.x == 0) a.moved[0] = 0;
}

// Thinning streams, first step: one block per request counts what stays, finds the first dropped token and lists where the rows
// that stay are now.
__global__ void __launch_bounds__(kKeepThreads) cache_keep_kernel(const BookArgs a) {
  __shared__ long long warp_sum[32];
  __shared__ int lowest, whole;
  chained_wait();
  chained_next();
  const int i = blockIdx.x;
  if (threadIdx.x == 0) lowest = 0x7fffffff;
  const int s = a.streams[i];
  bool bad = s < 0 || s >= a.n_streams;
  for (int j = threadIdx.x; j < i; j += blockDim.x) bad = bad || a.streams[j] == s;
  if (__syncthreads_or(bad) != 0) {
    if (threadIdx.x == 0) a.kept[i] = -1;
    return;
  }
  const int len = stream_length(a, s), held = pages_of(len, a.page);
  const int* row = a.table + s * a.width;
  for (int c = threadIdx.x; c < held; c += blockDim.x) a.old_pages[i * a.width + c] = row[c];
  const uint8_t* keep = a.keep + i * a.keep_stride;
  int2* moves = a.moves + i * a.moves_cap;
  constexpr int kEach = 16;                                                // neighbouring tokens per thread and turn
  int before = 0;
  for (long long t0 = 0; t0 < len; t0 += kEach * kKeepThreads) {
    const long long t = t0 + kEach * threadIdx.x;
    unsigned bits = 0, there = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (t + e < len) {
        there |= 1u << e;
        if (t + e < a.keep_stride && keep[t + e] != 0) bits |= 1u << e;
      }
    const unsigned dropped = there & ~bits;
    const int drop = __reduce_min_sync(0xffffffffu, dropped != 0 ? (int)(t + __ffs(dropped) - 1) : 0x7fffffff);
    if ((threadIdx.x & 31) == 0 && drop != 0x7fffffff) atomicMin(&lowest, drop);
    const int mine = __popc(bits), upto = block_scan<int>(mine, warp_sum);
    int at = before + upto - mine;
    // 16 tokens may span two pages (a page holds whole groups of 16, and t is a multiple of 16: they do not)
    const int page = bits != 0 ? row[t / a.page] : -1;
    const int place = page >= 0 && page < a.n_pages ? page * a.page + (int)(t % a.page) : -1;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if ((bits >> e) & 1u) moves[at++].x = place >= 0 ? place + e : -1;
    if (threadIdx.x == blockDim.x - 1) whole = upto;
    __syncthreads();
    before += whole;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    a.kept[i] = before;
    a.first[i] = lowest < len ? lowest : len;
  }
}

// Second step: the pages before the one with the first dropped token stay; new pages take the rest of what stays, and the old ones
// lose a holder once all requests have been served (so that no row is written while it may still be read).
__global__ void __launch_bounds__(kBookThreads) cache_compact_kernel(const BookArgs a) {
  extern __shared__ __align__(16) unsigned char book_raw[];
  BookSmem& sm = *reinterpret_cast<BookSmem*>(book_raw);
  int* begin = sm.extra;                                   // the first page that does not stay
  chained_wait();
  chained_next();
  load_streams(a, sm);
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    int need = -1, st = kCacheBadStream;
    begin[i] = 0;
    const int kept = a.kept[i];
    if (kept >= 0) {
      const int first = a.first[i];
      begin[i] = first / a.page;
      if (kept == first) {
        // a prefix stays: nothing moves, unless a page that becomes partly filled is another stream's, too
        const int p = first % a.page != 0 ? a.old_pages[i * a.width + first / a.page] : -1;
        if (p < 0 || p >= a.n_pages || a.refs[p] <= 1) begin[i] = pages_of(first, a.page);
      }
      need = max(0, pages_of(kept, a.page) - begin[i]);
      st = kCacheOk;
    }
    sm.need[i] = need;
    if (a.status != nullptr) a.status[i] = st;
  }
  const Served served = allocate(a, sm, [&](int i, int k, int p) { a.table[sm.streams[i] * a.width + begin[i] + k] = p; });
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < a.n; i += blockDim.x >> 5) {
    if (!served(sm, i)) continue;
    const long long s = sm.streams[i];
    const int held = pages_of(stream_length(a, s), a.page);
    for (int c = begin[i] + lane; c < held; c += 32) {
      const int p = a.old_pages[i * a.width + c];
      if (p >= 0 && p < a.n_pages) atomicSub(a.refs + p, 1);
      if (c >= begin[i] + sm.need[i]) a.table[s * a.width + c] = -1;
    }
    __syncwarp();
    if (lane == 0) a.lens[s] = a.kept[i];
  }
  __syncthreads();
  // rows to copy before request i, and the token that the copy of a request starts from
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    sm.need[i] = sm.need[i] > 0 && served(sm, i) ? a.kept[i] - begin[i] * a.page : 0;
    a.first[i] = begin[i] * a.page;
  }
  __syncthreads();
  sum_up(a, sm, [&](int i) { return sm.need[i]; });
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) a.moved[i + 1] = sm.ends[i];
  if (threadIdx.x == 0) a.moved[0] = 0;
}

// ---------------------------------------------------------------------------------------------
// Copies rows from page to page, in all layers, K and V.  Bound by HBM: 98 us for 0.624 GB read and written (4 streams, up to
// 3,120 rows each, 8 layers x 8 heads x 128), 6.4 TB/s; 400 whole pages of 64 tokens, 1.68 GB: 264 us, as much.  A warp takes one row of one layer: its K and V (kv_heads * head_dim values
// each) in 16-byte chunks, eight loads in flight.
// ---------------------------------------------------------------------------------------------
struct MoveArgs {
  __nv_bfloat16* k;
  __nv_bfloat16* v;
  long long ks[4], vs[4];       // element strides {layer, page, token, head}
  int layers, page, kv_heads, head_dim;
  long long n_pages;
  int n;
  // rows chosen by the bookkeeping ...
  const int2* moves;
  long long moves_cap;
  const long long* moved;
  const int* first;             // compact: destinations follow from the new table; fork: nullptr, they are in the list
  const int* streams;
  const int* table;
  long long width;
  // ... or whole pages, as the caller lists them
  const int* src_pages;
  const int* dst_pages;
};

template <bool kPages>
__global__ void __launch_bounds__(256) cache_move_kernel(const MoveArgs a) {
  chained_wait();
  chained_next();
  const int lane = threadIdx.x & 31;
  const long long rows = kPages ? (long long)a.n * a.page : a.moved[a.n];
  const long long items = rows * a.layers;
  const long long warps = (long long)gridDim.x * (blockDim.x >> 5);
  const int chunks = a.head_dim >> 3, row_chunks = a.kv_heads * chunks;
  for (long long it = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); it < items; it += warps) {
    const long long r = it % rows;
    const int layer = (int)(it / rows);
    long long from_page, to_page;
    int from_row, to_row;
    if (kPages) {
      const int i = (int)(r / a.page);
      from_page = a.src_pages[i];
      to_page = a.dst_pages[i];
      from_row = to_row = (int)(r % a.page);
      if (from_page == to_page) continue;
    } else {
      int lo = 0, hi = a.n - 1;                                            // the request this row belongs to
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.moved[mid + 1] > r) hi = mid; else lo = mid + 1;
      }
      const long long k = r - a.moved[lo];
      int src, dst;
      if (a.first != nullptr) {
        const long long j = a.first[lo] + k;
        src = a.moves[lo * a.moves_cap + j].x;
        dst = a.table[a.streams[lo] * a.width + j / a.page] * a.page + (int)(j % a.page);
      } else {
        const int2 m = a.moves[lo * a.moves_cap + k];
        src = m.x;
        dst = m.y;
      }
      if (src < 0) continue;                                               // (the old table named no page there)
      from_page = src / a.page; from_row = src % a.page;
      to_page = dst / a.page;   to_row = dst % a.page;
    }
    if (from_page < 0 || from_page >= a.n_pages || to_page < 0 || to_page >= a.n_pages) continue;
    const __nv_bfloat16* ksrc = a.k + layer * a.ks[0] + from_page * a.ks[1] + from_row * a.ks[2];
    const __nv_bfloat16* vsrc = a.v + layer * a.vs[0] + from_page * a.vs[1] + from_row * a.vs[2];
    __nv_bfloat16* kdst = a.k + layer * a.ks[0] + to_page * a.ks[1] + to_row * a.ks[2];
    __nv_bfloat16* vdst = a.v + layer * a.vs[0] + to_page * a.vs[1] + to_row * a.vs[2];
    for (int c0 = 0; c0 < row_chunks; c0 += 4 * 32) {
      uint4 x[4], y[4];
      long long ko[4], vo[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = c0 + u * 32 + lane, h = c / chunks, e = (c % chunks) * 8;
        ko[u] = h * a.ks[3] + e;
        vo[u] = h * a.vs[3] + e;
        if (c < row_chunks) {
          x[u] = *reinterpret_cast<const uint4*>(ksrc + ko[u]);
          y[u] = *reinterpret_cast<const uint4*>(vsrc + vo[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (c0 + u * 32 + lane < row_chunks) {
          *reinterpret_cast<uint4*>(kdst + ko[u]) = x[u];
          *reinterpret_cast<uint4*>(vdst + vo[u]) = y[u];
        }
    }
  }
}

}  // namespace sol
