// A K/V cache in pages: bringing new tokens in (norm, rotation, write), and opening, growing, thinning and closing streams.
//
// A cache is [layers][pages][page][kv_heads][head_dim]; token j of a stream is row j % page of page table[stream][j / page], in every
// layer.  refs[p] counts the streams that hold page p; a page is free while it is 0.  A page that several streams hold is full
// and never written again: forking shares full pages and copies the last, partly filled one at once.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "device_types.cuh"

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

// Tokens of a stream that the table has room for.
__device__ __forceinline__ long long stream_tokens(const PagedDev& c, long long stream) {
  const long long n = c.lens[stream], cap = c.width * c.page;
  return n < 0 ? 0 : n < cap ? n : cap;
}

// ---------------------------------------------------------------------------------------------
// New tokens of a plan's sequences into one layer of a cache: K and (optionally) Q are RMS-normalised per head, rotated by
// the token's (t, h, w), offset per sequence, and rounded once; V is copied.  Row i of a chunk of n tokens becomes token
// N - n + i of a stream of N.  Bound by HBM: every value is read and written once.
//
// A thread owns a 16-byte chunk (8 dims) of a token's rows: Q heads, then K heads, then V heads, `blockDim.x / chunks` rows
// apart, four of them in flight.  The angles of its four pairs are found once per token: from the plan's tables, or, where
// positions are offset, as position times frequency in fp64 (the tables end with the grid, and fp32 loses far positions), which
// B200 does at half its fp32 rate.
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
  double omega[64];             // frequency of pair j of head_dim / 2, 0 where nothing rotates
};

__global__ void __launch_bounds__(256, 3) cache_append_kernel(const __grid_constant__ AppendArgs a) {
  __shared__ int found;
  const int D = a.g.head_dim, chunks = D >> 3;
  const int rows_per_pass = blockDim.x / chunks;
  const int chunk = threadIdx.x % chunks, sub = threadIdx.x / chunks;
  const unsigned lanes = __activemask();
  const float inv_d = 1.0f / (float)D;
  const int n_q = a.x[0] != nullptr ? a.g.heads : 0, n_k = a.c.kv_heads, n_rows = n_q + 2 * n_k;
  constexpr int kBatch = 4;

  for (long long tok = blockIdx.x; tok < a.total_tokens; tok += gridDim.x) {
    for (int s = threadIdx.x; s < a.n_seqs; s += blockDim.x)
      if (tok >= a.seqs[s].tok_start && tok < a.seqs[s].tok_start + a.seqs[s].n_tokens) found = s;
    __syncthreads();
    const SeqDev sq = a.seqs[found];
    __syncthreads();
    const int local = (int)(tok - sq.tok_start);
    const long long stream = a.streams != nullptr ? a.streams[sq.seq_id] : sq.seq_id;
    if (stream < 0 || stream >= a.c.n_streams) continue;                   // an idle sequence (the same for the whole block)
    // Of several sequences with one stream the first counts: they would write the same rows.
    bool again = false;
    if (a.streams != nullptr) {
      for (int s = threadIdx.x; s < sq.seq_id; s += blockDim.x) again = again || a.streams[s] == stream;
      again = __syncthreads_or(again) != 0;
    }
    const long long at = stream_tokens(a.c, stream) - sq.n_tokens + local;
    long long page = -1;
    if (at >= 0 && !again) page = a.c.table[stream * a.c.width + at / a.c.page];
    const bool write = page >= 0 && page < a.c.n_pages;                    // (a table that names no page there: nothing is written)
    const int in_page = write ? (int)(at % a.c.page) : 0;
    const bool rotate = local >= sq.text_len;
    float2 cs[4];
    if (rotate) {
      const int p = local - sq.text_len, hw = sq.H * sq.W;
      const int pos[3] = {p / hw, (p / sq.W) % sq.H, p % sq.W};
      const int d1 = a.g.rope[0], d2 = d1 + a.g.rope[1], d3 = d2 + a.g.rope[2];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int d = chunk * 8 + 2 * u;                                   // first head dim of the pair
        const int axis = d < d1 ? 0 : d < d2 ? 1 : 2;
        const int x = axis == 0 ? pos[0] : axis == 1 ? pos[1] : pos[2];
        if (d >= d3) {
          cs[u] = make_float2(1.f, 0.f);
        } else if (a.pos0 != nullptr) {
          double s, c;
          sincos((double)((long long)x + a.pos0[3 * sq.seq_id + axis]) * a.omega[d >> 1], &s, &c);
          cs[u] = make_float2((float)c, (float)s);
        } else {
          const int first = axis == 0 ? 0 : axis == 1 ? d1 : d2;
          cs[u] = __ldg(&a.tables[a.g.tab_off[axis] + x * (a.g.rope[axis] >> 1) + ((d - first) >> 1)]);
        }
      }
    }
    for (int r0 = 0; r0 < n_rows; r0 += kBatch * rows_per_pass) {          // the same trip count for every thread
      uint4 w[kBatch];
      int which[kBatch], head[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int r = r0 + sub + b * rows_per_pass;
        which[b] = r < n_q ? 0 : r < n_q + n_k ? 1 : r < n_rows ? 2 : 3;
        head[b] = which[b] == 0 ? r : which[b] == 1 ? r - n_q : r - n_q - n_k;
        if (which[b] < 3) {
          const long long x_tok = which[b] == 0 ? a.x_tok[0] : which[b] == 1 ? a.x_tok[1] : a.x_tok[2];
          const long long x_head = which[b] == 0 ? a.x_head[0] : which[b] == 1 ? a.x_head[1] : a.x_head[2];
          const __nv_bfloat16* x = which[b] == 0 ? a.x[0] : which[b] == 1 ? a.x[1] : a.x[2];
          w[b] = __ldg(reinterpret_cast<const uint4*>(x + tok * x_tok + head[b] * x_head + chunk * 8));
        } else {
          w[b] = make_uint4(0, 0, 0, 0);
        }
      }
      float rinv[kBatch];
      if (a.gain[0] != nullptr || a.gain[1] != nullptr) {
        // Sums of squares of the rows, by shuffles over a row's chunks; where they leave fp32's range, once more on scaled values.
        auto squares = [&](float scale, float (&ss)[kBatch]) {
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            const uint32_t x[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
            ss[b] = 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const float lo = __uint_as_float(x[u] << 16) * scale, hi = __uint_as_float(x[u] & 0xffff0000u) * scale;
              ss[b] = fmaf(lo, lo, ss[b]);
              ss[b] = fmaf(hi, hi, ss[b]);
            }
          }
          for (int off = chunks >> 1; off > 0; off >>= 1)
#pragma unroll
            for (int b = 0; b < kBatch; ++b) ss[b] += __shfl_xor_sync(lanes, ss[b], off);
        };
        float ss[kBatch];
        squares(1.0f, ss);
        bool large = false, small = false;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          rinv[b] = rsqrtf(ss[b] * inv_d + a.eps);
          large = large || !(ss[b] < 1e37f);
          small = small || (ss[b] < 1e-25f && a.eps < 1e-20f);
        }
        if (__any_sync(lanes, large)) {
          float s2[kBatch];
          squares(0x1p-70f, s2);
#pragma unroll
          for (int b = 0; b < kBatch; ++b)                                 // 2^-70 is a factor of the root; eps is beside 1e37 / D nothing
            if (!(ss[b] < 1e37f)) rinv[b] = rsqrtf(s2[b] * inv_d + a.eps * 0x1p-120f * 0x1p-20f) * 0x1p-70f;
        }
        if (__any_sync(lanes, small)) {
          float s2[kBatch];
          squares(0x1p60f, s2);
#pragma unroll
          for (int b = 0; b < kBatch; ++b)
            if (ss[b] < 1e-25f && a.eps < 1e-20f) rinv[b] = rsqrtf(s2[b] * inv_d + a.eps * 0x1p120f) * 0x1p60f;
        }
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        if (which[b] == 3) break;
        uint4 y = w[b];
        if (which[b] < 2) {
          const uint32_t x[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
          float f[8];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            f[2 * u] = __uint_as_float(x[u] << 16);
            f[2 * u + 1] = __uint_as_float(x[u] & 0xffff0000u);
          }
          const float* gain = which[b] == 0 ? a.gain[0] : a.gain[1];
          if (gain != nullptr) {
            const float4 g0 = __ldg(reinterpret_cast<const float4*>(gain + chunk * 8));
            const float4 g1 = __ldg(reinterpret_cast<const float4*>(gain + chunk * 8) + 1);
            const float r = rinv[b];
            f[0] = f[0] * r * g0.x; f[1] = f[1] * r * g0.y; f[2] = f[2] * r * g0.z; f[3] = f[3] * r * g0.w;
            f[4] = f[4] * r * g1.x; f[5] = f[5] * r * g1.y; f[6] = f[6] * r * g1.z; f[7] = f[7] * r * g1.w;
          }
          if (rotate) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              if (cs[u].x == 1.f && cs[u].y == 0.f) continue;              // (keeps infinities in dims that do not rotate)
              const float re = f[2 * u], ro = f[2 * u + 1];
              f[2 * u] = re * cs[u].x - ro * cs[u].y;
              f[2 * u + 1] = re * cs[u].y + ro * cs[u].x;
            }
          }
          y = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        }
        if (which[b] == 0) {
          *reinterpret_cast<uint4*>(a.q_out + (tok * a.g.heads + head[b]) * (long long)D + chunk * 8) = y;
        } else if (write) {
          __nv_bfloat16* dst = which[b] == 1 ? a.c.k + page * a.c.ks[0] + in_page * a.c.ks[1] + head[b] * a.c.ks[2]
                                             : a.c.v + page * a.c.vs[0] + in_page * a.c.vs[1] + head[b] * a.c.vs[2];
          *reinterpret_cast<uint4*>(dst + chunk * 8) = y;
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Bookkeeping of streams and pages.  Requests of one call are served in their order: those that are in order take the free
// pages of the lowest index one after another, and a request that would need more than are left gets none.  Everything is
// integer arithmetic whose result does not depend on the order in which threads run.
// ---------------------------------------------------------------------------------------------
enum : int { kCacheOk = 0, kCacheBadStream = 1, kCacheNoRoom = 2, kCacheNoPages = 3, kCacheNotEmpty = 4 };
constexpr int kMaxRequests = 4096;
constexpr int kBookThreads = 1024;

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
// Is the stream of request i there, and not named by an earlier request?
__device__ __forceinline__ bool named_first(const BookArgs& a, int i) {
  const int s = a.streams[i];
  if (s < 0 || s >= a.n_streams) return false;
  for (int j = 0; j < i; ++j)
    if (a.streams[j] == s) return false;
  return true;
}

// Inclusive sums over the block's threads; `warp_sum` has 32 entries.  All threads call it.
__device__ __forceinline__ long long block_scan(long long x, long long* warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sum[warp] = x;
  __syncthreads();
  if (warp == 0) {
    long long t = lane < (int)(blockDim.x >> 5) ? warp_sum[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += y;
    }
    warp_sum[lane] = t;
  }
  __syncthreads();
  if (warp > 0) x += warp_sum[warp - 1];
  __syncthreads();
  return x;
}

struct BookSmem {
  long long warp_sum[32];
  long long ends[kMaxRequests];  // need of the requests up to and including i
  int need[kMaxRequests];        // pages, or -1: refused
};

// Turns need[] into running sums and refuses what does not fit the free pages; returns the number of pages to hand out.
__device__ __forceinline__ long long admit(const BookArgs& a, BookSmem& sm) {
  long long wanted = 0;
  for (int i0 = 0; i0 < a.n; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    const long long x = i < a.n && sm.need[i] > 0 ? sm.need[i] : 0;
    const long long s = block_scan(x, sm.warp_sum);
    if (i < a.n) sm.ends[i] = wanted + s;
    __syncthreads();
    wanted = sm.ends[min(i0 + (int)blockDim.x, a.n) - 1];
  }
  return wanted;
}

// Hands out `wanted` free pages, lowest index first: calls give(request, k, page) for the k-th page of a request.  Returns how many
// there were.  A request gets all its pages or none: admit_found below says which.
template <typename Give>
__device__ __forceinline__ long long hand_out(const BookArgs& a, BookSmem& sm, long long wanted, const Give& give) {
  long long found = 0;
  for (long long p0 = 0; p0 < a.n_pages && found < wanted; p0 += blockDim.x) {
    const long long p = p0 + threadIdx.x;
    const bool is_free = p < a.n_pages && a.refs[p] == 0;
    const long long rank = block_scan(is_free ? 1 : 0, sm.warp_sum) - 1 + found;        // among all free pages
    if (is_free && rank < wanted) {
      int lo = 0, hi = a.n - 1;                                            // the first request whose running sum exceeds the rank
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sm.ends[mid] > rank) hi = mid; else lo = mid + 1;
      }
      give(lo, (int)(rank - (sm.ends[lo] - sm.need[lo])), (int)p);
    }
    found += __syncthreads_count(is_free);
  }
  return found < wanted ? found : wanted;
}
// The free pages are counted first (up to what is wanted), so that a request that cannot be served takes none.
__device__ __forceinline__ long long count_free(const BookArgs& a, long long wanted) {
  long long found = 0;
  for (long long p0 = 0; p0 < a.n_pages && found < wanted; p0 += 8ll * blockDim.x) {
    int mine = 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const long long p = p0 + u * (long long)blockDim.x + threadIdx.x;
      mine += p < a.n_pages && a.refs[p] == 0 ? 1 : 0;
    }
    // 0 .. 8 free pages per thread: four counts of one bit
#pragma unroll
    for (int bit = 0; bit < 4; ++bit) found += (long long)__syncthreads_count((mine >> bit) & 1) << bit;
  }
  return found;
}

// Closing streams: their pages lose a holder.
__global__ void __launch_bounds__(kBookThreads) cache_free_kernel(const BookArgs a) {
  __shared__ int ok[kMaxRequests];
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    ok[i] = named_first(a, i);
    if (a.status != nullptr) a.status[i] = ok[i] ? kCacheOk : kCacheBadStream;
  }
  __syncthreads();
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < a.n; i += blockDim.x >> 5) {
    if (!ok[i]) continue;
    const long long s = a.streams[i];
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
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    int need = -1, st = kCacheBadStream;
    if (named_first(a, i) && a.amount[i] >= 0) {
      const int len = stream_length(a, a.streams[i]);
      const long long want = (long long)len + a.amount[i];
      st = kCacheNoRoom;
      if (want <= a.width * a.page && want <= 0x7fffffffll) {
        st = kCacheOk;
        need = pages_of((int)want, a.page) - pages_of(len, a.page);
      }
    }
    sm.need[i] = need;
    if (a.status != nullptr) a.status[i] = st;
  }
  __syncthreads();
  const long long wanted = admit(a, sm), there = count_free(a, wanted);
  for (int i = threadIdx.x; i < a.n; i += blockDim.x)
    if (sm.need[i] > 0 && sm.ends[i] > there) {
      if (a.status != nullptr) a.status[i] = kCacheNoPages;
    }
  __syncthreads();
  hand_out(a, sm, wanted < there ? wanted : there, [&](int i, int k, int p) {
    if (sm.ends[i] > there) return;
    const long long s = a.streams[i];
    a.table[s * a.width + pages_of(stream_length(a, s), a.page) + k] = p;
    a.refs[p] = 1;
  });
  __syncthreads();
  for (int i = threadIdx.x; i < a.n; i += blockDim.x)
    if (sm.need[i] >= 0 && !(sm.need[i] > 0 && sm.ends[i] > there)) a.lens[a.streams[i]] = stream_length(a, a.streams[i]) + a.amount[i];
}

// Opening streams as branches of others: full pages are shared, the last, partly filled one is copied (by cache_move_kernel).
__global__ void __launch_bounds__(kBookThreads) cache_fork_kernel(const BookArgs a) {
  extern __shared__ __align__(16) unsigned char book_raw[];
  BookSmem& sm = *reinterpret_cast<BookSmem*>(book_raw);
  int* len = reinterpret_cast<int*>(book_raw + sizeof(BookSmem));          // of the parents, before anything changes
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    int st = kCacheBadStream, need = -1;
    const int parent = a.parents[i];
    len[i] = 0;
    if (named_first(a, i) && parent >= 0 && parent < a.n_streams) {
      st = kCacheNotEmpty;
      if (stream_length(a, a.streams[i]) == 0) {
        st = kCacheOk;
        len[i] = stream_length(a, parent);
        need = len[i] % a.page != 0 ? 1 : 0;
      }
    }
    sm.need[i] = need;
    if (a.status != nullptr) a.status[i] = st;
  }
  __syncthreads();
  const long long wanted = admit(a, sm), there = count_free(a, wanted);
  for (int i = threadIdx.x; i < a.n; i += blockDim.x)
    if (sm.need[i] > 0 && sm.ends[i] > there) {
      if (a.status != nullptr) a.status[i] = kCacheNoPages;
    }
  __syncthreads();
  hand_out(a, sm, wanted < there ? wanted : there, [&](int i, int k, int p) {
    if (sm.ends[i] > there) return;
    a.table[a.streams[i] * a.width + len[i] / a.page] = p;
    a.refs[p] = 1;
  });
  __syncthreads();
  // one warp per request: the shared pages, and which rows of the last one have to be copied
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < a.n; i += blockDim.x >> 5) {
    if (sm.need[i] < 0 || (sm.need[i] > 0 && sm.ends[i] > there)) continue;
    const long long s = a.streams[i], parent = a.parents[i];
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
  // rows to copy before request i
  long long before = 0;
  for (int i0 = 0; i0 < a.n; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    long long x = 0;
    if (i < a.n && sm.need[i] > 0 && sm.ends[i] <= there) x = len[i] % a.page;
    const long long s = block_scan(x, sm.warp_sum);
    if (i < a.n) {
      a.moved[i + 1] = before + s;
      sm.ends[i] = before + s;
    }
    __syncthreads();
    before = sm.ends[min(i0 + (int)blockDim.x, a.n) - 1];
  }
  if (threadIdx.x == 0) a.moved[0] = 0;
}

// Thinning streams, first step: one block per request counts what stays, finds the first dropped token and lists where the rows
// that stay are now.
__global__ void __launch_bounds__(kBookThreads) cache_keep_kernel(const BookArgs a) {
  __shared__ long long warp_sum[32];
  __shared__ int in_order;
  __shared__ int lowest;
  const int i = blockIdx.x;
  if (threadIdx.x == 0) lowest = 0x7fffffff;
  {
    const int s = a.streams[i];
    bool bad = s < 0 || s >= a.n_streams;
    for (int j = threadIdx.x; j < i; j += blockDim.x) bad = bad || a.streams[j] == s;
    bad = __syncthreads_or(bad) != 0;
    if (threadIdx.x == 0) in_order = !bad;
  }
  __syncthreads();
  if (!in_order) {
    if (threadIdx.x == 0) a.kept[i] = -1;
    return;
  }
  const long long s = a.streams[i];
  const int len = stream_length(a, s), held = pages_of(len, a.page);
  const int* row = a.table + s * a.width;
  for (int c = threadIdx.x; c < held; c += blockDim.x) a.old_pages[i * a.width + c] = row[c];
  const uint8_t* keep = a.keep + i * a.keep_stride;
  constexpr int kEach = 8;                                                 // neighbouring tokens per thread and turn
  long long before = 0;
  for (long long t0 = 0; t0 < len; t0 += kEach * kBookThreads) {
    const long long t = t0 + kEach * threadIdx.x;
    unsigned bits = 0;
    int drop = 0x7fffffff;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (t + e < len) {
        if (t + e < a.keep_stride && keep[t + e] != 0) bits |= 1u << e;
        else if (drop == 0x7fffffff) drop = (int)(t + e);
      }
    drop = __reduce_min_sync(0xffffffffu, drop);
    if ((threadIdx.x & 31) == 0 && drop != 0x7fffffff) atomicMin(&lowest, drop);
    const int mine = __popc(bits);
    const long long upto = block_scan(mine, warp_sum);
    long long at = before + upto - mine;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if ((bits >> e) & 1u) {
        const int p = row[(t + e) / a.page];
        a.moves[i * a.moves_cap + at++].x = p >= 0 && p < a.n_pages ? p * a.page + (int)((t + e) % a.page) : -1;
      }
    if (threadIdx.x == blockDim.x - 1) warp_sum[0] = upto;
    __syncthreads();
    before += warp_sum[0];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    a.kept[i] = (int)before;
    a.first[i] = lowest < len ? lowest : len;
  }
}

// Second step: the pages before the one with the first dropped token stay; new pages take the rest of what stays, and the old ones
// lose a holder once all requests have been served (so that no row is written while it may still be read).
__global__ void __launch_bounds__(kBookThreads) cache_compact_kernel(const BookArgs a) {
  extern __shared__ __align__(16) unsigned char book_raw[];
  BookSmem& sm = *reinterpret_cast<BookSmem*>(book_raw);
  int* begin = reinterpret_cast<int*>(book_raw + sizeof(BookSmem));        // the first page that does not stay
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    int need = -1, st = kCacheBadStream;
    begin[i] = 0;
    if (a.kept[i] >= 0) {
      const int kept = a.kept[i], first = a.first[i];
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
  __syncthreads();
  const long long wanted = admit(a, sm), there = count_free(a, wanted);
  auto served = [&](int i) { return sm.need[i] >= 0 && !(sm.need[i] > 0 && sm.ends[i] > there); };
  for (int i = threadIdx.x; i < a.n; i += blockDim.x)
    if (sm.need[i] > 0 && !served(i) && a.status != nullptr) a.status[i] = kCacheNoPages;
  __syncthreads();
  hand_out(a, sm, wanted < there ? wanted : there, [&](int i, int k, int p) {
    if (sm.ends[i] > there) return;
    a.table[a.streams[i] * a.width + begin[i] + k] = p;
    a.refs[p] = 1;
  });
  __syncthreads();
  const int lane = threadIdx.x & 31;
  for (int i = threadIdx.x >> 5; i < a.n; i += blockDim.x >> 5) {
    if (!served(i)) continue;
    const long long s = a.streams[i];
    const int held = pages_of(stream_length(a, s), a.page);
    for (int c = begin[i] + lane; c < held; c += 32) {
      const int p = a.old_pages[i * a.width + c];
      if (p >= 0 && p < a.n_pages) atomicSub(a.refs + p, 1);
      if (c >= begin[i] + sm.need[i]) a.table[s * a.width + c] = -1;
    }
    __syncwarp();
    if (lane == 0) a.lens[s] = a.kept[i];
  }
  long long before = 0;
  for (int i0 = 0; i0 < a.n; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    long long x = 0;
    if (i < a.n && sm.need[i] > 0 && served(i)) x = a.kept[i] - (long long)begin[i] * a.page;
    if (i < a.n) a.first[i] = begin[i] * a.page;                           // what the copying kernel starts from
    __syncthreads();
    const long long sum = block_scan(x, sm.warp_sum);
    if (i < a.n) a.moved[i + 1] = before + sum;
    __syncthreads();
    before = a.moved[min(i0 + (int)blockDim.x, a.n)];
  }
  if (threadIdx.x == 0) a.moved[0] = 0;
}

// ---------------------------------------------------------------------------------------------
// Copies rows from page to page, in all layers, K and V.  Bound by HBM.  A warp takes one row of one layer: its K and V
// (kv_heads * head_dim values each) in 16-byte chunks, eight loads in flight.
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
