// Host side of streaming generation: paged cache, attention over it, cross attention.  Part of sol_attn3d.cu (inside extern "C").

extern "C++" {
namespace {

bool aligned4(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 3u) == 0; }

// Raises a kernel's limit of dynamic shared memory, once per device.
template <auto kKernel>
cudaError_t allow_shared_memory(int bytes) {
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  else (void)cudaGetLastError();
  return e;
}

// Launches a kernel that begins with chained_wait(): it may be placed on the GPU while its predecessor in the stream still runs.
template <typename... Params, typename... Args>
cudaError_t launch_chained(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, const Args&... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  if (e != cudaSuccess) (void)cudaGetLastError();
  return e;
}

// Keys are counted in 32 bits, and the kernels look a tile or a page past them.
constexpr long long kMaxKeys = (1ll << 31) - 8192;

// Checks a cache and, for a layer, fills in what the kernels see of it.
int take_cache(const sol_attn3d_paged_cache* c, int layer, sol::PagedDev* out) {
  if (c == nullptr || c->size != sizeof(sol_attn3d_paged_cache) || c->n_layers < 1 || c->page_size < 1 || c->kv_heads < 1 ||
      c->head_dim < 1 || c->n_pages < 1 || c->n_streams < 1 || c->table_width < 1 || layer < 0 || layer >= c->n_layers)
    return SOL_ATTN3D_ERR_INVALID_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->kv_heads > 65535 || c->page_size % 16 != 0 || c->page_size > 4096 ||
      c->n_pages >= (1ll << 31) || c->table_width >= (1ll << 31) || c->n_streams >= (1ll << 31) ||
      c->n_pages * c->page_size > kMaxKeys || c->table_width * c->page_size > kMaxKeys)
    return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  if (c->k == nullptr || c->v == nullptr || c->table == nullptr || c->lens == nullptr || !aligned16(c->k) || !aligned16(c->v) ||
      !aligned4(c->table) || !aligned4(c->lens) || !aligned4(c->refs))
    return SOL_ATTN3D_ERR_INVALID_ARG;
  auto take = [&](const int64_t st[4], long long (&full)[4]) {
    full[3] = st[3] == 0 ? c->head_dim : st[3];
    full[2] = st[2] == 0 ? (long long)c->kv_heads * c->head_dim : st[2];
    if (!stride_ok(full[3]) || !stride_ok(full[2])) return false;
    full[1] = st[1] == 0 ? c->page_size * full[2] : st[1];
    if (!stride_ok(full[1])) return false;
    full[0] = st[0] == 0 ? c->n_pages * full[1] : st[0];
    return full[0] > 0 && full[0] % 8 == 0 && full[0] < (1ll << 46);
  };
  long long ks[4], vs[4];
  if (!take(c->k_strides, ks) || !take(c->v_strides, vs)) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  out->k = static_cast<__nv_bfloat16*>(c->k) + layer * ks[0];
  out->v = static_cast<__nv_bfloat16*>(c->v) + layer * vs[0];
  for (int i = 0; i < 3; ++i) {
    out->ks[i] = ks[i + 1];
    out->vs[i] = vs[i + 1];
  }
  out->table = c->table;
  out->lens = c->lens;
  out->width = c->table_width;
  out->n_streams = c->n_streams;
  out->n_pages = c->n_pages;
  out->page = c->page_size;
  out->kv_heads = c->kv_heads;
  return SOL_ATTN3D_OK;
}

int take_context(const sol_attn3d_context* x, sol::KeysDev* d) {
  if (x == nullptr || x->size != sizeof(sol_attn3d_context) || x->kv_heads < 1 || x->head_dim < 1 || x->total_rows < 0 || x->max_len < 0)
    return SOL_ATTN3D_ERR_INVALID_ARG;
  if ((x->head_dim != 64 && x->head_dim != 128) || x->kv_heads > 65535 || x->total_rows > kMaxKeys)
    return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  if (x->begins == nullptr || x->lens == nullptr || !aligned4(x->begins) || !aligned4(x->lens) || !aligned16(x->k) || !aligned16(x->v) ||
      (x->total_rows > 0 && (x->k == nullptr || x->v == nullptr)))
    return SOL_ATTN3D_ERR_INVALID_ARG;
  auto take = [&](const int64_t st[2], long long (&full)[3]) {
    full[0] = 0;
    full[2] = st[1] == 0 ? x->head_dim : st[1];
    full[1] = st[0] == 0 ? (long long)x->kv_heads * x->head_dim : st[0];
    return stride_ok(full[1]) && stride_ok(full[2]);
  };
  if (!take(x->k_strides, d->c.ks) || !take(x->v_strides, d->c.vs)) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  d->c.k = static_cast<__nv_bfloat16*>(const_cast<void*>(x->k));
  d->c.v = static_cast<__nv_bfloat16*>(const_cast<void*>(x->v));
  d->c.kv_heads = x->kv_heads;
  d->begins = x->begins;
  d->lens = x->lens;
  d->total_rows = x->total_rows;
  d->mask = x->key_mask;
  return SOL_ATTN3D_OK;
}

// ---- attention of few rows ------------------------------------------------------------------------------------------------
// Splits of the keys: about 1,024 keys of the longest possible past per CTA, so that streams of different length even out; at least
// a wave of resident CTAs when there are few units, at most eight waves (a table may be far wider than its streams are long, and a
// CTA without keys still costs its start); never below 256 keys.  Depends on the sizes of the call only (the lengths live on the
// device).
constexpr long long kFewWave = 148 * sol::kFewResident, kFewMinKeys = 256, kFewMaxSplit = 256;
int few_splits(long long items, long long capacity) {
  if (items < 1) return 1;
  const long long want = std::min(std::max((capacity + 1023) / 1024, kFewWave / items), (8 * kFewWave + items - 1) / items);
  return (int)std::max<long long>(1, std::min(std::min(want, kFewMaxSplit), capacity / kFewMinKeys));
}
long long few_units(sol_attn3d_plan_t p, int batch, int group) {
  return p != nullptr ? p->total_tokens * group / sol::kFewRows + p->n_seqs : (long long)batch * ((group + sol::kFewRows - 1) / sol::kFewRows);
}
size_t few_bytes(long long units, int kv_heads, int head_dim, long long capacity) {
  const int n = few_splits(units * kv_heads, capacity);
  return n == 1 ? 0 : align_up((size_t)units * kv_heads * n * sol::kFewRows * (head_dim + 4) * sizeof(float));
}

template <int D, bool kPaged>
cudaError_t launch_few(const sol::FewArgs& f, int rows, cudaStream_t st, int* launches) {
  const unsigned items = (unsigned)(f.units * f.d.c.kv_heads);
  cudaError_t e = allow_shared_memory<&sol::few_rows_kernel<D, kPaged>>(sol::FewSmem<D>::kBytes);
  if (e != cudaSuccess) return e;
  if ((e = launch_chained(sol::few_rows_kernel<D, kPaged>, items * (unsigned)f.n_split, sol::kFewThreads, sol::FewSmem<D>::kBytes, st, f)) != cudaSuccess) return e;
  ++*launches;
  if (f.partial != nullptr) {
    const bool shared = f.n_split > 8;                     // a row's parts over the CTA's warps, or a warp per row: see join_few_kernel
    e = shared ? launch_chained(sol::join_few_kernel<D, kPaged, sol::kJoinFewWarps>, dim3(items, (unsigned)rows), 32 * sol::kJoinFewWarps, 0, st, f)
               : launch_chained(sol::join_few_kernel<D, kPaged, 1>, dim3(items, (unsigned)(rows + sol::kJoinFewWarps - 1) / sol::kJoinFewWarps),
                                32 * sol::kJoinFewWarps, 0, st, f);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

// Attention of `units` units of few rows; plan or batch as in few_units, no sequence of more than `longest` tokens.
int attend_few(sol::QueriesDev a, const sol::KeysDev& d, bool paged, int head_dim, long long units, long long longest, long long capacity,
               void* workspace, size_t workspace_bytes, cudaStream_t st, int* launches, cudaError_t* cuda_error) {
  sol::FewArgs f{};
  f.a = a;
  f.d = d;
  f.units = units;
  f.n_split = few_splits(units * d.c.kv_heads, capacity);
  if (units * d.c.kv_heads * f.n_split >= (1ll << 31)) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  if (f.n_split > 1) {
    if (workspace == nullptr || workspace_bytes < few_bytes(units, d.c.kv_heads, head_dim, capacity) ||
        (reinterpret_cast<uintptr_t>(workspace) % kAlign) != 0)
      return SOL_ATTN3D_ERR_NO_WORKSPACE;
    f.partial = static_cast<float*>(workspace);
  }
  const int rows = (int)std::min<long long>(sol::kFewRows, longest * a.group);
  *cuda_error = head_dim == 128 ? (paged ? launch_few<128, true>(f, rows, st, launches) : launch_few<128, false>(f, rows, st, launches))
                                : (paged ? launch_few<64, true>(f, rows, st, launches) : launch_few<64, false>(f, rows, st, launches));
  return *cuda_error == cudaSuccess ? SOL_ATTN3D_OK : SOL_ATTN3D_ERR_CUDA;
}

// ---- attention over a plan's sequences ---------------------------------------------------------------------------------------
constexpr size_t kUnitCounterOffset = 128;   // next unit of context_attn_kernel inside the 256-byte status block of a workspace

// How a plan's rows are served for `kv_heads` K/V heads and pasts of up to `capacity` keys.  Few rows per K/V head (one unit of
// few_rows_kernel in every sequence) go to that kernel, more to the tensor-core kernel, whose tile is 128 rows high.  Both kernels, 40 / 8
// heads x 128: 24 streams of 200 to 11,700 keys, 15 rows each 120 and 165 us, 20 rows 175 and 166; one stream of 111,856 keys, 5 rows 98
// and 106, 15 rows 111 and 106, 20 rows 177 and 107; 40 / 40 heads, 24 streams, 12 rows 482 and 600, 20 rows 810 and 573.
struct ContextRoute {
  bool few;
  int group, tok_per_tile, n_split;
  long long units;              // per K/V head
  long long n_whole, n_tail;    // more than kSortedSeqs sequences: units of all heads that take all of their keys; units whose keys are split
  long long max_parts, max_joins;   // what the workspace has room for
};
ContextRoute choose_route(sol_attn3d_plan_t p, int kv_heads, long long capacity, long long total_rows) {
  ContextRoute r{};
  r.group = p->heads / kv_heads;
  const long long longest = p->sched.front().n_tokens;
  r.few = longest * r.group <= sol::kFewRows || r.group > 128 || total_rows == 0;
  if (r.few) {
    r.units = few_units(p, 0, r.group);
    r.n_split = few_splits(r.units * kv_heads, capacity);
    return r;
  }
  r.tok_per_tile = 128 / r.group;
  const int per_unit = 2 * r.tok_per_tile;
  const long long tiles = (capacity + 127) / 128;
  if (p->n_seqs <= sol::kSortedSeqs) {
    // planned on the device: room for three waves of parts, or for all that units of four key tiles at least can make
    for (const SeqDev& q : p->sched) r.units += (q.n_tokens + per_unit - 1) / per_unit;
    r.n_split = 1;
    r.n_whole = r.units * kv_heads;
    const long long parts = std::min<long long>(32, tiles / 4);
    if (parts >= 2) r.max_parts = std::min<long long>(3 * sol::kPlanSms, r.n_whole * parts);
    r.max_joins = r.max_parts / 2;
    return r;
  }
  // Many sequences: what is left after the last whole wave of units, or all of them if there are few, is split so that it ends as one
  // wave of short units; the longest possible past is assumed.  Costs as in context_attn_kernel.
  r.units = p->total_tokens / per_unit + p->n_seqs;
  const long long flat = r.units * kv_heads, waves = flat / sol::kPlanSms;
  double best = 0.0;
  for (int n = 1; n <= std::max<long long>(1, std::min<long long>(32, tiles / 4)); ++n) {
    const long long whole = waves * sol::kPlanSms, tail = flat - whole;
    const double cost = (double)waves * (tiles + 2.0) + (double)((tail * n + sol::kPlanSms - 1) / sol::kPlanSms) * ((tiles + n - 1) / n + 2.0) +
                        (n > 1 ? 1.5 + 0.03 * (double)(tail * n) : 0.0);
    if (n == 1 || cost < best) {
      best = cost;
      r.n_split = n;
      r.n_whole = n > 1 ? whole : flat;
      r.n_tail = flat - r.n_whole;
    }
  }
  if (r.n_tail == 0) r.n_split = 1;
  if (r.n_split > 1) {
    r.max_parts = r.n_tail * r.n_split;
    r.max_joins = r.n_tail;
  }
  return r;
}

size_t join_list_bytes(const ContextRoute& r) { return kAlign + align_up((size_t)r.max_joins * sizeof(sol::JoinUnit)); }

size_t many_bytes(const ContextRoute& r, int head_dim) {
  return r.max_parts == 0 ? 0 : join_list_bytes(r) + align_up((size_t)r.max_parts * 2 * r.tok_per_tile * r.group * (head_dim + 4) * sizeof(float));
}

size_t context_bytes(sol_attn3d_plan_t p, int kv_heads, long long capacity, long long total_rows) {
  if (p == nullptr || p->heads % kv_heads != 0) return 0;
  const ContextRoute r = choose_route(p, kv_heads, capacity, total_rows);
  return r.few ? few_bytes(r.units, kv_heads, p->head_dim, capacity) : many_bytes(r, p->head_dim);
}

// Any tensor as a tiled map of bf16 boxes 64 elements wide, 128-byte swizzle; strides of the outer dimensions in elements.
int encode_boxes(sol_attn3d_plan_t p, CUtensorMap* tm, const void* base, int rank, const long long* dims, const long long* strides, const int* box) {
  cuuint64_t d[4], s[3];
  cuuint32_t b[4];
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    d[i] = (cuuint64_t)dims[i];
    b[i] = (cuuint32_t)box[i];
    if (i > 0) s[i - 1] = (cuuint64_t)strides[i - 1] * 2;
  }
  const CUresult r = p->encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d, s, b, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r == CUDA_SUCCESS) return SOL_ATTN3D_OK;
  p->last_cuda = (int)r;
  return SOL_ATTN3D_ERR_CUDA;
}

template <int D, bool kPaged, bool kMask, bool kBoxes>
cudaError_t launch_context_as(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& o, const sol::ContextParams& c, long long items,
                             int sms, cudaStream_t st, int* launches) {
  cudaError_t e = allow_shared_memory<&sol::context_attn_kernel<D, kPaged, kMask, kBoxes>>(sol::ContextSmem<D>::kDynBytes);
  if (e != cudaSuccess) return e;
  if ((e = launch_chained(sol::context_attn_kernel<D, kPaged, kMask, kBoxes>, (unsigned)std::min<long long>(items, sms), sol::kAttnThreads, sol::ContextSmem<D>::kDynBytes, st,
                          q, k, v, o, c)) != cudaSuccess) return e;
  ++*launches;
  if (c.partial != nullptr) {
    const sol::JoinArgs j{c.a, 2 * c.tok_per_tile * c.a.group, c.partial, c.join, c.join_count, c.status};
    if ((e = launch_chained(sol::join_units_kernel<D>, 4 * sol::kPlanSms, 32 * sol::kJoinWarps, 0, st, j)) != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

template <int D, bool kPaged>
cudaError_t launch_context(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& o, const sol::ContextParams& c, long long items, int sms,
                           cudaStream_t st, int* launches) {
  if constexpr (!kPaged)
    if (32 % c.a.group == 0)                               // a warp's 32 rows are whole tokens: a box of o
      return c.d.mask != nullptr ? launch_context_as<D, false, true, true>(q, k, v, o, c, items, sms, st, launches)
                                 : launch_context_as<D, false, false, true>(q, k, v, o, c, items, sms, st, launches);
  return c.d.mask != nullptr ? launch_context_as<D, kPaged, true, false>(q, k, v, o, c, items, sms, st, launches)
                             : launch_context_as<D, kPaged, false, false>(q, k, v, o, c, items, sms, st, launches);
}

int attend_many(sol_attn3d_plan_t p, const sol::QueriesDev& a, const sol::KeysDev& d, bool paged, const ContextRoute& r, void* workspace,
                size_t workspace_bytes, cudaStream_t st) {
  sol::ContextParams c{};
  c.a = a;
  c.d = d;
  c.units = r.units;
  c.n_split = r.n_split;
  c.n_whole = r.n_whole;
  c.n_tail = r.n_tail;
  const long long items = r.n_whole + r.n_tail * r.n_split + r.max_parts;   // at most (the grid need not be larger; the counter has to hold them)
  if (items >= (1ll << 31)) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  c.max_parts = (int)r.max_parts;
  c.tok_per_tile = r.tok_per_tile;
  c.inv_group = (65536u + r.group - 1) / r.group;
  if (r.max_parts > 0) {
    if (workspace == nullptr || workspace_bytes < many_bytes(r, p->head_dim) || (reinterpret_cast<uintptr_t>(workspace) % kAlign) != 0) return SOL_ATTN3D_ERR_NO_WORKSPACE;
    c.join_count = static_cast<int*>(workspace);
    c.join = reinterpret_cast<sol::JoinUnit*>(static_cast<unsigned char*>(workspace) + kAlign);
    c.partial = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + join_list_bytes(r));
  }
  c.counter = reinterpret_cast<unsigned int*>(p->ws + p->off_status + kUnitCounterOffset);
  c.status = reinterpret_cast<unsigned int*>(p->ws + p->off_status);
  c.rescales = reinterpret_cast<unsigned int*>(p->ws + p->off_status + kCountersOffset);
  c.wait_limit_ns = p->wait_limit_ns;
  c.fault_inject = p->fault_inject;
  c.v_lbo = p->v_lbo;
  c.v_sbo = p->v_sbo;
  CUtensorMap tm_q, tm_k, tm_v, tm_o;
  const long long q_dims[3] = {p->head_dim, p->heads, p->total_tokens}, q_strides[2] = {a.q_head, a.q_tok};
  const int q_box[3] = {64, r.group, r.tok_per_tile};
  int rc = encode_boxes(p, &tm_q, a.q, 3, q_dims, q_strides, q_box);
  tm_o = tm_q;                                             // (not looked at, unless rows are written by boxes)
  if (rc == SOL_ATTN3D_OK && !paged && 32 % r.group == 0) {
    const long long o_strides[2] = {a.o_head, a.o_tok};
    const int o_box[3] = {64, r.group, 32 / r.group};
    rc = encode_boxes(p, &tm_o, a.out, 3, q_dims, o_strides, o_box);
  }
  for (int kv = 0; kv < 2 && rc == SOL_ATTN3D_OK; ++kv) {
    CUtensorMap* tm = kv ? &tm_v : &tm_k;
    const void* base = kv ? d.c.v : d.c.k;
    const long long* s = kv ? d.c.vs : d.c.ks;
    if (paged) {
      c.box_rows = 16;
      while (c.box_rows < 128 && d.c.page % (2 * c.box_rows) == 0) c.box_rows *= 2;
      const long long dims[4] = {p->head_dim, d.c.kv_heads, d.c.page, d.c.n_pages}, strides[3] = {s[2], s[1], s[0]};
      const int box[4] = {64, 1, c.box_rows, 1};
      rc = encode_boxes(p, tm, base, 4, dims, strides, box);
    } else {
      c.box_rows = 128;
      const long long dims[3] = {p->head_dim, d.c.kv_heads, d.total_rows}, strides[2] = {s[2], s[1]};
      const int box[3] = {64, 1, 128};
      rc = encode_boxes(p, tm, base, 3, dims, strides, box);
    }
  }
  if (rc != SOL_ATTN3D_OK) return rc;
  const cudaError_t e = p->head_dim == 128 ? (paged ? launch_context<128, true>(tm_q, tm_k, tm_v, tm_o, c, items, p->sm_count, st, &p->launches)
                                                    : launch_context<128, false>(tm_q, tm_k, tm_v, tm_o, c, items, p->sm_count, st, &p->launches))
                                           : (paged ? launch_context<64, true>(tm_q, tm_k, tm_v, tm_o, c, items, p->sm_count, st, &p->launches)
                                                    : launch_context<64, false>(tm_q, tm_k, tm_v, tm_o, c, items, p->sm_count, st, &p->launches));
  return e == cudaSuccess ? SOL_ATTN3D_OK : fail_cuda(p, e);
}

int forward_context(sol_attn3d_plan_t p, const void* q, void* out, const sol::KeysDev& d, bool paged, long long capacity, int causal,
                    void* workspace, size_t workspace_bytes, sol_attn3d_stream_t stream) {
  if (q == nullptr || out == nullptr || q == out || !aligned16(q) || !aligned16(out)) return SOL_ATTN3D_ERR_INVALID_ARG;
  if (p->heads % d.c.kv_heads != 0) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  const long long total_rows = paged ? 1 : d.total_rows;
  const ContextRoute r = choose_route(p, d.c.kv_heads, capacity, total_rows);
  if ((long long)p->sched.front().n_tokens * r.group >= (1ll << 31)) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;   // rows are counted in 32 bits
  if (p->ws == nullptr || p->encode == nullptr) return SOL_ATTN3D_ERR_NO_WORKSPACE;
  sol::QueriesDev a{};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.q_tok = p->sq.tok; a.q_head = p->sq.head;
  a.o_tok = p->so.tok; a.o_head = p->so.head;
  a.seqs = reinterpret_cast<const SeqDev*>(p->ws + p->off_seqs);
  a.cum_tok = reinterpret_cast<const int*>(p->ws + p->off_cum);
  a.n_seqs = p->n_seqs;
  a.group = r.group;
  a.causal = causal;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)p->head_dim));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  p->launches = 0;
  if (p->prof) {                                           // no bits and no rotary prologue: only the last interval counts
    p->prof_valid = false;
    p->prof_bits = false;
    for (int i = 0; i < 3; ++i)
      if ((e = cudaEventRecord(p->ev[i], st)) != cudaSuccess) return fail_cuda(p, e);
  }
  e = cudaSuccess;
  const int rc = r.few ? attend_few(a, d, paged, p->head_dim, r.units, p->sched.front().n_tokens, capacity, workspace, workspace_bytes, st, &p->launches, &e)
                       : attend_many(p, a, d, paged, r, workspace, workspace_bytes, st);
  if (e != cudaSuccess) return fail_cuda(p, e);
  if (rc != SOL_ATTN3D_OK) return rc;
  if (p->prof) {
    if ((e = cudaEventRecord(p->ev[3], st)) != cudaSuccess) return fail_cuda(p, e);
    p->prof_valid = true;
  }
  return SOL_ATTN3D_OK;
}

int step_context(const void* q, const int64_t q_strides[2], const sol::KeysDev& d, bool paged, void* out, const int64_t out_strides[2],
                 int batch, int heads, int head_dim, long long capacity, void* workspace, size_t workspace_bytes, sol_attn3d_stream_t stream) {
  if (batch < 0 || heads < 1) return SOL_ATTN3D_ERR_INVALID_ARG;
  if (heads % d.c.kv_heads != 0 || heads > 65535) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  if (batch == 0) return SOL_ATTN3D_OK;
  if (q == nullptr || out == nullptr || q == out || !aligned16(q) || !aligned16(out) || q_strides == nullptr || out_strides == nullptr)
    return SOL_ATTN3D_ERR_INVALID_ARG;
  sol::QueriesDev a{};
  const long long row = (long long)heads * head_dim;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.q_tok = q_strides[0] == 0 ? row : q_strides[0];
  a.q_head = q_strides[1] == 0 ? head_dim : q_strides[1];
  a.o_tok = out_strides[0] == 0 ? row : out_strides[0];
  a.o_head = out_strides[1] == 0 ? head_dim : out_strides[1];
  if (!stride_ok(a.q_tok) || !stride_ok(a.q_head) || !stride_ok(a.o_tok) || !stride_ok(a.o_head)) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  a.n_seqs = batch;
  a.group = heads / d.c.kv_heads;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)head_dim));
  int launches = 0;                                        // (a plan counts them)
  cudaError_t e = cudaSuccess;
  const int rc = attend_few(a, d, paged, head_dim, few_units(nullptr, batch, a.group), 1, capacity, workspace, workspace_bytes,
                            static_cast<cudaStream_t>(stream), &launches, &e);
  return e != cudaSuccess ? planless_status(e) : rc;
}

size_t step_bytes(int batch, int heads, int kv_heads, int head_dim, long long capacity) {
  if (batch < 1 || heads < 1 || heads % kv_heads != 0) return 0;
  return few_bytes(few_units(nullptr, batch, heads / kv_heads), kv_heads, head_dim, capacity);
}

// ---- bookkeeping --------------------------------------------------------------------------------------------------------------
// Workspace of fork and compact: moves [n][capacity] | moved [n + 1] | kept [n] | first [n] | old_pages [n][table_width]
struct BookSpace {
  size_t moved, kept, first, old_pages, bytes;
};
BookSpace book_space(const sol_attn3d_paged_cache* c, int n) {
  BookSpace s;
  size_t o = align_up((size_t)n * c->table_width * c->page_size * sizeof(int2));
  s.moved = o;     o = align_up(o + ((size_t)n + 1) * sizeof(long long));
  s.kept = o;      o = align_up(o + (size_t)n * sizeof(int));
  s.first = o;     o = align_up(o + (size_t)n * sizeof(int));
  s.old_pages = o; o = align_up(o + (size_t)n * c->table_width * sizeof(int));
  s.bytes = o;
  return s;
}

int take_book(const sol_attn3d_paged_cache* c, int n, const int32_t* streams, int32_t* status, sol::BookArgs* b) {
  sol::PagedDev layer{};
  const int rc = take_cache(c, 0, &layer);
  if (rc != SOL_ATTN3D_OK) return rc;
  if (n < 0 || c->refs == nullptr || !aligned4(streams) || !aligned4(status) || (n > 0 && streams == nullptr)) return SOL_ATTN3D_ERR_INVALID_ARG;
  if (n > sol::kMaxRequests) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  b->table = c->table;
  b->lens = c->lens;
  b->refs = c->refs;
  b->width = c->table_width;
  b->n_streams = c->n_streams;
  b->n_pages = c->n_pages;
  b->page = c->page_size;
  b->n = n;
  b->streams = streams;
  b->status = status;
  return SOL_ATTN3D_OK;
}

int take_book_space(const sol_attn3d_paged_cache* c, int n, void* workspace, size_t bytes, sol::BookArgs* b) {
  const BookSpace s = book_space(c, n);
  if (workspace == nullptr || bytes < s.bytes || (reinterpret_cast<uintptr_t>(workspace) % kAlign) != 0) return SOL_ATTN3D_ERR_NO_WORKSPACE;
  unsigned char* w = static_cast<unsigned char*>(workspace);
  b->moves = reinterpret_cast<int2*>(w);
  b->moves_cap = c->table_width * c->page_size;
  b->moved = reinterpret_cast<long long*>(w + s.moved);
  b->kept = reinterpret_cast<int*>(w + s.kept);
  b->first = reinterpret_cast<int*>(w + s.first);
  b->old_pages = reinterpret_cast<int*>(w + s.old_pages);
  return SOL_ATTN3D_OK;
}

constexpr size_t kBookSmem = sizeof(sol::BookSmem);

template <typename K>
int launch_book(K kernel, const sol::BookArgs& b, cudaStream_t st) {
  static_assert(kBookSmem <= 48 * 1024, "what a launch may have without being asked for");
  return planless_status(launch_chained(kernel, 1, sol::kBookThreads, kBookSmem, st, b));
}

template <bool kPages>
int launch_move(const sol_attn3d_paged_cache* c, sol::MoveArgs m, cudaStream_t st) {
  sol::PagedDev layer{};
  int rc = take_cache(c, 0, &layer);
  if (rc != SOL_ATTN3D_OK) return rc;
  m.k = layer.k;
  m.v = layer.v;
  for (int i = 0; i < 3; ++i) {
    m.ks[i + 1] = layer.ks[i];
    m.vs[i + 1] = layer.vs[i];
  }
  m.ks[0] = c->k_strides[0] == 0 ? c->n_pages * m.ks[1] : c->k_strides[0];
  m.vs[0] = c->v_strides[0] == 0 ? c->n_pages * m.vs[1] : c->v_strides[0];
  m.layers = c->n_layers;
  m.page = c->page_size;
  m.kv_heads = c->kv_heads;
  m.head_dim = c->head_dim;
  m.n_pages = c->n_pages;
  // the number of rows is on the device: eight resident blocks per SM walk over them
  return planless_status(launch_chained(sol::cache_move_kernel<kPages>, 148 * 8, 256, 0, st, m));
}

}  // namespace
}  // extern "C++"

size_t sol_attn3d_cache_workspace_bytes(const sol_attn3d_paged_cache* cache, int n) {
  sol::PagedDev layer{};
  if (n < 1 || n > sol::kMaxRequests || take_cache(cache, 0, &layer) != SOL_ATTN3D_OK) return 0;
  return book_space(cache, n).bytes;
}

int sol_attn3d_cache_reserve(const sol_attn3d_paged_cache* cache, int n, const int32_t* streams, const int32_t* amount, int32_t* status,
                             sol_attn3d_stream_t stream) {
  sol::BookArgs b{};
  const int rc = take_book(cache, n, streams, status, &b);
  if (rc != SOL_ATTN3D_OK || n == 0) return rc;
  if (amount == nullptr || !aligned4(amount)) return SOL_ATTN3D_ERR_INVALID_ARG;
  b.amount = amount;
  return launch_book(sol::cache_reserve_kernel, b, static_cast<cudaStream_t>(stream));
}

int sol_attn3d_cache_fork(const sol_attn3d_paged_cache* cache, int n, const int32_t* parents, const int32_t* streams, int32_t* status,
                          void* workspace, size_t workspace_bytes, sol_attn3d_stream_t stream) {
  sol::BookArgs b{};
  int rc = take_book(cache, n, streams, status, &b);
  if (rc != SOL_ATTN3D_OK || n == 0) return rc;
  if (parents == nullptr || !aligned4(parents)) return SOL_ATTN3D_ERR_INVALID_ARG;
  if ((rc = take_book_space(cache, n, workspace, workspace_bytes, &b)) != SOL_ATTN3D_OK) return rc;
  b.parents = parents;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if ((rc = launch_book(sol::cache_fork_kernel, b, st)) != SOL_ATTN3D_OK) return rc;
  sol::MoveArgs m{};
  m.n = n;
  m.moves = b.moves;
  m.moves_cap = b.moves_cap;
  m.moved = b.moved;
  return launch_move<false>(cache, m, st);
}

int sol_attn3d_cache_compact(const sol_attn3d_paged_cache* cache, int n, const int32_t* streams, const uint8_t* keep, int64_t keep_width,
                             int32_t* status, void* workspace, size_t workspace_bytes, sol_attn3d_stream_t stream) {
  sol::BookArgs b{};
  int rc = take_book(cache, n, streams, status, &b);
  if (rc != SOL_ATTN3D_OK || n == 0) return rc;
  if (keep == nullptr || keep_width < 1) return SOL_ATTN3D_ERR_INVALID_ARG;
  if ((rc = take_book_space(cache, n, workspace, workspace_bytes, &b)) != SOL_ATTN3D_OK) return rc;
  b.keep = keep;
  b.keep_stride = keep_width;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if ((rc = planless_status(launch_chained(sol::cache_keep_kernel, (unsigned)n, sol::kKeepThreads, 0, st, b))) != SOL_ATTN3D_OK) return rc;
  if ((rc = launch_book(sol::cache_compact_kernel, b, st)) != SOL_ATTN3D_OK) return rc;
  sol::MoveArgs m{};
  m.n = n;
  m.moves = b.moves;
  m.moves_cap = b.moves_cap;
  m.moved = b.moved;
  m.first = b.first;
  m.streams = streams;
  m.table = cache->table;
  m.width = cache->table_width;
  return launch_move<false>(cache, m, st);
}

int sol_attn3d_cache_free(const sol_attn3d_paged_cache* cache, int n, const int32_t* streams, int32_t* status, sol_attn3d_stream_t stream) {
  sol::BookArgs b{};
  const int rc = take_book(cache, n, streams, status, &b);
  if (rc != SOL_ATTN3D_OK || n == 0) return rc;
  return launch_book(sol::cache_free_kernel, b, static_cast<cudaStream_t>(stream));
}

int sol_attn3d_cache_copy_pages(const sol_attn3d_paged_cache* cache, int n, const int32_t* src_pages, const int32_t* dst_pages,
                                sol_attn3d_stream_t stream) {
  sol::PagedDev layer{};
  const int rc = take_cache(cache, 0, &layer);
  if (rc != SOL_ATTN3D_OK) return rc;
  if (n < 0) return SOL_ATTN3D_ERR_INVALID_ARG;
  if (n > (1 << 20)) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  if (n == 0) return SOL_ATTN3D_OK;
  if (src_pages == nullptr || dst_pages == nullptr || !aligned4(src_pages) || !aligned4(dst_pages)) return SOL_ATTN3D_ERR_INVALID_ARG;
  sol::MoveArgs m{};
  m.n = n;
  m.src_pages = src_pages;
  m.dst_pages = dst_pages;
  return launch_move<true>(cache, m, static_cast<cudaStream_t>(stream));
}

int sol_attn3d_cache_append(sol_attn3d_plan_t p, const void* q, const void* k, const void* v, const int64_t k_strides[2],
                            const int64_t v_strides[2], void* q_out, const sol_attn3d_paged_cache* cache, int layer,
                            const int32_t* streams, const int32_t* pos0, const float* q_gain, const float* k_gain, float eps,
                            sol_attn3d_stream_t stream) {
  if (p == nullptr || k == nullptr || v == nullptr || k_strides == nullptr || v_strides == nullptr) return SOL_ATTN3D_ERR_INVALID_ARG;
  if ((q == nullptr) != (q_out == nullptr) || (q != nullptr && (q == q_out || k == q_out || v == q_out))) return SOL_ATTN3D_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(q_gain) || !aligned16(k_gain) || !aligned4(streams) ||
      !aligned4(pos0) || !(eps >= 0.f) || !std::isfinite(eps))
    return SOL_ATTN3D_ERR_INVALID_ARG;
  sol::AppendArgs a{};
  const int rc = take_cache(cache, layer, &a.c);
  if (rc != SOL_ATTN3D_OK) return rc;
  if (cache->head_dim != p->head_dim) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  const long long dense = (long long)cache->kv_heads * cache->head_dim;
  const int64_t* st[2] = {k_strides, v_strides};
  a.x_tok[0] = p->sq.tok;
  a.x_head[0] = p->sq.head;
  for (int i = 0; i < 2; ++i) {
    a.x_tok[i + 1] = st[i][0] == 0 ? dense : st[i][0];
    a.x_head[i + 1] = st[i][1] == 0 ? cache->head_dim : st[i][1];
    if (!stride_ok(a.x_tok[i + 1]) || !stride_ok(a.x_head[i + 1])) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  }
  for (long long st : {a.x_head[0], a.x_head[1], a.x_head[2], a.c.ks[2], a.c.vs[2]})
    if (st > 0x7fffffffll) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  if (p->ws == nullptr) return SOL_ATTN3D_ERR_NO_WORKSPACE;
  a.x[0] = static_cast<const __nv_bfloat16*>(q);
  a.x[1] = static_cast<const __nv_bfloat16*>(k);
  a.x[2] = static_cast<const __nv_bfloat16*>(v);
  a.q_out = static_cast<__nv_bfloat16*>(q_out);
  a.gain[0] = q_gain;
  a.gain[1] = k_gain;
  a.eps = eps;
  a.seqs = reinterpret_cast<const SeqDev*>(p->ws + p->off_seqs);
  a.n_seqs = p->n_seqs;
  a.total_tokens = p->total_tokens;
  a.tables = reinterpret_cast<const float2*>(p->ws + p->off_tables);
  for (int i = 0; i < 3; ++i) { a.g.rope[i] = p->rope[i]; a.g.tab_off[i] = p->tab_off[i]; }
  a.g.head_dim = p->head_dim;
  a.g.heads = p->heads;
  a.streams = streams;
  a.pos0 = pos0;
  a.omega = reinterpret_cast<const double*>(p->ws + p->off_omega);
  const int chunks = p->head_dim / 8, rows = std::max(q != nullptr ? p->heads : 0, (int)cache->kv_heads);
  const int unit = 32 / chunks;                            // rows per warp
  const bool many = p->total_tokens >= 148 * 3 * 4;        // four tokens at a time, unless that leaves SMs idle
  const int per_pass = std::min(256 / chunks, ((many ? rows : (rows + 3) / 4) + unit - 1) / unit * unit);
  const long long blocks = std::min<long long>((p->total_tokens + (many ? 3 : 0)) / (many ? 4 : 1), 148ll * 3 * 8);
  p->launches = 0;
  const cudaError_t e = launch_chained(p->head_dim == 128 ? (many ? sol::cache_append_kernel<128, 4> : sol::cache_append_kernel<128, 1>)
                                                          : (many ? sol::cache_append_kernel<64, 4> : sol::cache_append_kernel<64, 1>),
                                       (unsigned)blocks, (unsigned)(chunks * per_pass), 0, static_cast<cudaStream_t>(stream), a);
  if (e != cudaSuccess) return fail_cuda(p, e);
  ++p->launches;
  return SOL_ATTN3D_OK;
}

size_t sol_attn3d_paged_workspace_bytes(sol_attn3d_plan_t plan, const sol_attn3d_paged_cache* cache) {
  sol::PagedDev c{};
  if (plan == nullptr || take_cache(cache, 0, &c) != SOL_ATTN3D_OK) return 0;
  return context_bytes(plan, c.kv_heads, c.width * c.page, 1);
}

int sol_attn3d_forward_paged(sol_attn3d_plan_t p, const void* q, const sol_attn3d_paged_cache* cache, int layer, void* out,
                             const int32_t* streams, const uint8_t* key_mask, int64_t mask_width, int causal_block, void* workspace,
                             size_t workspace_bytes, sol_attn3d_stream_t stream) {
  if (p == nullptr || causal_block < 0 || (key_mask != nullptr && mask_width < 1) || !aligned4(streams)) return SOL_ATTN3D_ERR_INVALID_ARG;
  sol::KeysDev d{};
  const int rc = take_cache(cache, layer, &d.c);
  if (rc != SOL_ATTN3D_OK) return rc;
  if (cache->head_dim != p->head_dim) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  d.streams = streams;
  d.mask = key_mask;
  d.mask_stride = mask_width;
  return forward_context(p, q, out, d, true, d.c.width * d.c.page, causal_block, workspace, workspace_bytes, stream);
}

size_t sol_attn3d_paged_step_workspace_bytes(const sol_attn3d_paged_cache* cache, int batch, int heads) {
  sol::PagedDev c{};
  if (take_cache(cache, 0, &c) != SOL_ATTN3D_OK) return 0;
  return step_bytes(batch, heads, c.kv_heads, cache->head_dim, c.width * c.page);
}

int sol_attn3d_paged_step(const void* q, const int64_t q_strides[2], const sol_attn3d_paged_cache* cache, int layer, const int32_t* streams,
                          void* out, const int64_t out_strides[2], int batch, int heads, const uint8_t* key_mask, int64_t mask_width,
                          void* workspace, size_t workspace_bytes, sol_attn3d_stream_t stream) {
  if ((key_mask != nullptr && mask_width < 1) || !aligned4(streams)) return SOL_ATTN3D_ERR_INVALID_ARG;
  sol::KeysDev d{};
  const int rc = take_cache(cache, layer, &d.c);
  if (rc != SOL_ATTN3D_OK) return rc;
  d.streams = streams;
  d.mask = key_mask;
  d.mask_stride = mask_width;
  return step_context(q, q_strides, d, true, out, out_strides, batch, heads, cache->head_dim, d.c.width * d.c.page, workspace, workspace_bytes, stream);
}

size_t sol_attn3d_cross_workspace_bytes(sol_attn3d_plan_t plan, const sol_attn3d_context* context) {
  sol::KeysDev d{};
  if (plan == nullptr || take_context(context, &d) != SOL_ATTN3D_OK) return 0;
  return context_bytes(plan, context->kv_heads, std::min(context->max_len, context->total_rows), context->total_rows);
}

int sol_attn3d_forward_cross(sol_attn3d_plan_t p, const void* q, const sol_attn3d_context* context, void* out, void* workspace,
                             size_t workspace_bytes, sol_attn3d_stream_t stream) {
  if (p == nullptr) return SOL_ATTN3D_ERR_INVALID_ARG;
  sol::KeysDev d{};
  const int rc = take_context(context, &d);
  if (rc != SOL_ATTN3D_OK) return rc;
  if (context->head_dim != p->head_dim) return SOL_ATTN3D_ERR_UNSUPPORTED_SHAPE;
  return forward_context(p, q, out, d, false, std::min(context->max_len, context->total_rows), 0, workspace, workspace_bytes, stream);
}

size_t sol_attn3d_cross_step_workspace_bytes(const sol_attn3d_context* context, int batch, int heads) {
  sol::KeysDev d{};
  if (take_context(context, &d) != SOL_ATTN3D_OK) return 0;
  return step_bytes(batch, heads, context->kv_heads, context->head_dim, std::min(context->max_len, context->total_rows));
}

int sol_attn3d_cross_step(const void* q, const int64_t q_strides[2], const sol_attn3d_context* context, void* out, const int64_t out_strides[2],
                          int batch, int heads, void* workspace, size_t workspace_bytes, sol_attn3d_stream_t stream) {
  sol::KeysDev d{};
  const int rc = take_context(context, &d);
  if (rc != SOL_ATTN3D_OK) return rc;
  return step_context(q, q_strides, d, false, out, out_strides, batch, heads, context->head_dim, std::min(context->max_len, context->total_rows),
                      workspace, workspace_bytes, stream);
}
