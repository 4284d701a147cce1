// Validation, plans and launches of the calls on a cache in pages.  Part of calidrop.hip, whose error string and helpers it
// uses.
#pragma once

namespace {

int check_paged(const calidrop_paged_params* p) {
  if (!p) return fail(CALIDROP_EINVAL, "params is NULL");
  if (p->struct_size != sizeof(calidrop_paged_params))
    return fail(CALIDROP_EINVAL, "params.struct_size is %u, this library expects %zu", p->struct_size, sizeof(calidrop_paged_params));
  if (p->dtype != CALIDROP_BF16 && p->dtype != CALIDROP_FP32)
    return fail(CALIDROP_EUNSUPPORTED, "dtype %d is not CALIDROP_BF16 or CALIDROP_FP32", p->dtype);
  if (p->batch < 1) return fail(CALIDROP_EINVAL, "batch must be >= 1 (got %d)", p->batch);
  if (p->batch > 65535) return fail(CALIDROP_EUNSUPPORTED, "batch %d exceeds 65535", p->batch);
  if (p->n_q_heads < 1 || p->n_kv_heads < 1)
    return fail(CALIDROP_EINVAL, "head counts must be >= 1 (got %d query, %d KV)", p->n_q_heads, p->n_kv_heads);
  if (p->n_q_heads % p->n_kv_heads != 0)
    return fail(CALIDROP_ESHAPE, "n_q_heads %d is not a multiple of n_kv_heads %d", p->n_q_heads, p->n_kv_heads);
  if (p->n_q_heads / p->n_kv_heads > 16)
    return fail(CALIDROP_EUNSUPPORTED, "GQA group size %d exceeds 16", p->n_q_heads / p->n_kv_heads);
  if (p->n_q_heads > 65535) return fail(CALIDROP_EUNSUPPORTED, "n_q_heads %d exceeds 65535", p->n_q_heads);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(CALIDROP_EUNSUPPORTED, "head_dim %d is not 64 or 128", p->head_dim);
  if (p->page_size < 1 || p->n_pages < 1 || p->max_pages < 1)
    return fail(CALIDROP_EINVAL, "page_size, n_pages and max_pages must be >= 1 (got %d, %d, %d)", p->page_size, p->n_pages, p->max_pages);
  if (static_cast<double>(p->page_size) * p->n_pages * p->n_kv_heads >= 4294967296.0)
    return fail(CALIDROP_EUNSUPPORTED, "n_pages * n_kv_heads * page_size exceeds 2^32 rows");
  if (!(p->scale >= 0.f) || std::isinf(p->scale))
    return fail(CALIDROP_EINVAL, "scale must be finite and >= 0 (0 selects 1/sqrt(head_dim))");
  if (p->window < 0 || p->sinks < 0)
    return fail(CALIDROP_EINVAL, "window and sinks must be >= 0 (got %d, %d)", p->window, p->sinks);
  if (p->rot_dim < 0 || p->rot_dim > p->head_dim)
    return fail(CALIDROP_EINVAL, "rot_dim must lie in [0, head_dim] (got %d)", p->rot_dim);
  if (p->rot_dim % 16 != 0) return fail(CALIDROP_EUNSUPPORTED, "rot_dim %d is not a multiple of 16", p->rot_dim);
  if (p->rot_pairs != CALIDROP_ROT_HALVES && p->rot_pairs != CALIDROP_ROT_NEIGHBOURS)
    return fail(CALIDROP_EINVAL, "rot_pairs %d is no calidrop_rot_pairs", p->rot_pairs);
  return CALIDROP_OK;
}

int64_t paged_capacity(const calidrop_paged_params* p) { return static_cast<int64_t>(p->max_pages) * p->page_size; }

struct NamedPtr { const void* ptr; const char* name; };
template <int N>
int check_ptrs(const NamedPtr (&req)[N]) {
  for (const auto& r : req)
    if (!r.ptr) return fail(CALIDROP_EINVAL, "%s is NULL", r.name);
  for (const auto& r : req)
    if (!aligned16(r.ptr)) return fail(CALIDROP_EALIGN, "%s is not 16-byte aligned", r.name);
  return CALIDROP_OK;
}

// magic = ceil(2^shift / d) with shift = 31 + ceil(log2 d); see page_div
cd::PageDiv page_divisor(int d) {
  int bits = 0;
  while ((static_cast<int64_t>(1) << bits) < d) ++bits;
  const int shift = 31 + bits;
  return {static_cast<uint32_t>(((static_cast<uint64_t>(1) << shift) + d - 1) / d), shift};
}

cd::Pages pages_of(const calidrop_paged_params* p, const int32_t* table, int64_t stride) {
  cd::Pages pg{};
  pg.table = table; pg.table_stride = stride; pg.page_size = p->page_size; pg.n_pages = p->n_pages; pg.Hkv = p->n_kv_heads;
  pg.div = page_divisor(p->page_size);
  return pg;
}

// How an attention launch is cut up: rows (token, head of the group) of a workgroup, splits of the cache, tiles of a split.
// Up to 32 rows stream the cache from memory to registers; more share tiles of it in LDS, in bf16 (fp32 products are sixteen
// times slower than bf16 ones and wait for nothing).
struct PagedPlan { int rows, NS, tiles; };
constexpr int kPagedTile = 32;             // rows of a streamed tile, half those of a shared one
constexpr int kPagedRowsAtOnce = 65536;    // rows of all workgroups, up to which a call is split further
constexpr int kPagedMostSplits = 128;
constexpr int kPagedMostRows = 128;

// Rows of the longest cache that the queries of a call can see.
int64_t paged_rows_seen(const calidrop_paged_params* p, int64_t max_q_len, int64_t max_len) {
  if (!p->window) return max_len;
  return std::min<int64_t>(max_len, static_cast<int64_t>(p->window) + p->sinks + max_q_len);
}
// Most tiles of `tile` rows that a workgroup of `rows` can need (cd::KeyTiles): under a window, the rows of the window and of the
// sinks can begin and end inside a tile each, and share one.
int64_t most_tiles(const calidrop_paged_params* p, int64_t q_len, int64_t max_len, int64_t rows, int64_t tile) {
  const int64_t all = (max_len + tile - 1) / tile;
  if (!p->window) return all;
  const int64_t tokens = std::min(q_len, rows / (p->n_q_heads / p->n_kv_heads) + 2);
  return std::min(all + 1, (p->window + tokens + tile - 1) / tile + 1 + (p->sinks + tile - 1) / tile);
}
int most_paged_splits(int64_t seen) { return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kPagedMostSplits, (seen + 127) / 128))); }

PagedPlan plan_paged(const calidrop_paged_params* p, int64_t sequences, int64_t q_len, int64_t total_q, int64_t max_len) {
  const int64_t G = p->n_q_heads / p->n_kv_heads, rows = q_len * G;
  PagedPlan plan;
  plan.rows = rows <= 16 ? 16 : rows <= 32 || p->dtype == CALIDROP_FP32 ? 32 : kPagedMostRows;
  const bool shared = plan.rows == kPagedMostRows;
  const int64_t groups = p->n_kv_heads * std::max(sequences * ((rows + plan.rows - 1) / plan.rows), (total_q * G + plan.rows - 1) / plan.rows);
  const int64_t most = shared ? kPagedRowsAtOnce / plan.rows : 2048;
  const int64_t want = std::max<int64_t>(std::min<int64_t>(most_paged_splits(paged_rows_seen(p, q_len, max_len)), most / groups), 1);
  const int64_t tile = shared ? 2 * kPagedTile : kPagedTile, unit = shared ? 2 : 4;     // no fewer than 128 rows
  const int64_t tiles = most_tiles(p, q_len, max_len, plan.rows, tile);
  plan.tiles = static_cast<int>(std::max((((tiles + want - 1) / want) + unit - 1) / unit * unit, unit));
  plan.NS = static_cast<int>(std::max<int64_t>(1, (tiles + plan.tiles - 1) / plan.tiles));
  return plan;
}

// Room for the partials of `rows` (token, head) rows: splits of a call make kPagedRowsAtOnce rows at most.
size_t partial_rows(int64_t rows, int64_t seen) {
  return static_cast<size_t>(std::min<int64_t>(rows * most_paged_splits(seen), kPagedRowsAtOnce));
}
size_t partial_bytes(const calidrop_paged_params* p, size_t rows) {
  return round256(rows * sizeof(float2)) + round256(rows * p->head_dim * sizeof(float));
}
size_t attend_bytes(const calidrop_paged_params* p, int64_t total_q, int32_t max_q_len, int32_t max_cache_len) {
  return std::max<size_t>(256, partial_bytes(p, partial_rows(total_q * p->n_q_heads, paged_rows_seen(p, max_q_len, max_cache_len))));
}
size_t shared_bytes(const calidrop_paged_params* p, int64_t total_q, int32_t max_q_len, int32_t max_cache_len, int32_t shared_len) {
  const int64_t rows = total_q * p->n_q_heads;       // where a side is not split its partials are there all the same
  return std::max<size_t>(256, partial_bytes(p, 2 * rows + partial_rows(rows, paged_rows_seen(p, max_q_len, max_cache_len)) +
                                                    partial_rows(rows, shared_len)));
}

int check_attend_sizes(const calidrop_paged_params* p, int64_t total_q, int32_t max_q_len, int32_t max_cache_len) {
  if (total_q < 0 || max_q_len < 1 || max_cache_len < 0)
    return fail(CALIDROP_ESHAPE, "total_q >= 0, max_q_len >= 1 and max_cache_len >= 0 expected (got %lld, %d, %d)",
                static_cast<long long>(total_q), max_q_len, max_cache_len);
  if (total_q > (int64_t{1} << 30) / p->n_q_heads)
    return fail(CALIDROP_EUNSUPPORTED, "total_q * n_q_heads exceeds 2^30");
  if (max_q_len > (int64_t{1} << 30) / p->n_q_heads)
    return fail(CALIDROP_EUNSUPPORTED, "max_q_len * n_q_heads exceeds 2^30");
  if (max_cache_len > paged_capacity(p))
    return fail(CALIDROP_ESHAPE, "max_cache_len %d exceeds the max_pages * page_size = %lld rows of a table", max_cache_len,
                static_cast<long long>(paged_capacity(p)));
  if (max_cache_len > (1 << 30)) return fail(CALIDROP_EUNSUPPORTED, "max_cache_len %d exceeds 2^30", max_cache_len);
  return CALIDROP_OK;
}
int check_shared_sizes(const calidrop_paged_params* p, int32_t shared_len) {
  if (shared_len < 1) return fail(CALIDROP_ESHAPE, "shared_len must be >= 1 (got %d)", shared_len);
  if (shared_len > (1 << 30)) return fail(CALIDROP_EUNSUPPORTED, "shared_len %d exceeds 2^30", shared_len);
  if (p->window || p->sinks) return fail(CALIDROP_EUNSUPPORTED, "a shared prefix goes without window and sinks (got %d, %d)", p->window, p->sinks);
  return CALIDROP_OK;
}

template <typename T, int D>
int launch_paged(const cd::PagedAttendArgs& a, const PagedPlan& plan, int64_t sequences, int64_t q_len, hipStream_t st) {
  const int64_t rows = q_len * a.G, blocks = (rows + plan.rows - 1) / plan.rows;
  const dim3 grid(static_cast<unsigned>(blocks * plan.NS), a.pages.Hkv, static_cast<unsigned>(sequences));
  if constexpr (sizeof(T) == 2) {
    if (plan.rows == kPagedMostRows) {
      hipLaunchKernelGGL((cd::paged_tile_kernel<D>), grid, dim3(256), 0, st, a);
      return launch_status("paged_attend");
    }
  }
  if (plan.rows == 16) hipLaunchKernelGGL((cd::paged_stream_kernel<T, D, 1>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((cd::paged_stream_kernel<T, D, 2>), grid, dim3(256), 0, st, a);
  return launch_status("paged_attend");
}

// shared_table NULL: no prefix.
template <typename T, int D>
int attend_impl(const calidrop_paged_params* p, cd::PagedAttendArgs a, int32_t max_cache_len, const int32_t* shared_table,
                int32_t shared_len, char* ws, hipStream_t st) {
  const PagedPlan own = plan_paged(p, p->batch, a.max_q_len, a.total_q, max_cache_len);
  PagedPlan prefix{};
  if (shared_table) prefix = plan_paged(p, 1, a.total_q, a.total_q, shared_len);
  a.slots = own.NS + prefix.NS;
  a.part_ml = reinterpret_cast<float2*>(ws);
  a.part_o = reinterpret_cast<float*>(ws + round256(static_cast<size_t>(a.total_q) * a.Hq * a.slots * sizeof(float2)));
  int rc;
  if (shared_table) {
    cd::PagedAttendArgs f = a;
    f.pages.table = shared_table; f.pages.table_stride = 0; f.lens = nullptr; f.fixed_len = shared_len; f.max_len = shared_len;
    f.all_see_all = 1; f.slot0 = own.NS; f.NS = prefix.NS; f.tiles_per_split = prefix.tiles;
    if ((rc = launch_paged<T, D>(f, prefix, 1, a.total_q, st))) return rc;
  }
  a.NS = own.NS; a.tiles_per_split = own.tiles;
  if ((rc = launch_paged<T, D>(a, own, p->batch, a.max_q_len, st))) return rc;
  if (a.slots == 1) return CALIDROP_OK;
  static_assert(2 * kPagedMostSplits <= cd::kJoinSlots, "the joining waves hold every partial of a row");
  const int64_t rows = a.total_q * a.Hq;
  if (a.slots <= 8) hipLaunchKernelGGL((cd::paged_join_kernel<T, D, 1>), dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((cd::paged_join_kernel<T, D, 4>), dim3(static_cast<unsigned>(rows)), dim3(256), 0, st, a);
  return launch_status("paged_join");
}

int attend_entry(const calidrop_paged_params* p, const void* q, const int32_t* q_offsets, int64_t total_q, int32_t max_q_len,
                 const void* k_pages, const void* v_pages, const int32_t* shared_table, int32_t shared_len,
                 const int32_t* page_table, const int32_t* cache_lens, int32_t max_cache_len, void* out, float* lse,
                 void* workspace, size_t workspace_bytes, size_t need, void* stream) {
  int rc;
  if (!q_offsets && (total_q != p->batch))
    return fail(CALIDROP_ESHAPE, "without q_offsets every sequence has one token: total_q %lld is not the batch %d",
                static_cast<long long>(total_q), p->batch);
  if (total_q == 0) return CALIDROP_OK;
  if ((rc = check_ptrs({{q, "q"}, {k_pages, "k_pages"}, {v_pages, "v_pages"}, {page_table, "page_table"}, {cache_lens, "cache_lens"},
                        {out, "out"}, {lse, "lse"}}))) return rc;
  if (!aligned16(q_offsets)) return fail(CALIDROP_EALIGN, "q_offsets is not 16-byte aligned");
  if (!aligned16(shared_table)) return fail(CALIDROP_EALIGN, "shared_table is not 16-byte aligned");
  if (!workspace || workspace_bytes < need)
    return fail(CALIDROP_EWORKSPACE, "workspace of %zu bytes given, %zu needed", workspace ? workspace_bytes : 0, need);
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(CALIDROP_EALIGN, "workspace is not 256-byte aligned");
  cd::PagedAttendArgs a{};
  a.q = q; a.q_off = q_offsets; a.k = k_pages; a.v = v_pages; a.lens = cache_lens; a.max_len = max_cache_len;
  a.pages = pages_of(p, page_table, p->max_pages);
  a.total_q = total_q; a.batch = p->batch; a.Hq = p->n_q_heads; a.G = p->n_q_heads / p->n_kv_heads;
  a.max_q_len = q_offsets ? max_q_len : 1;
  a.window = std::min(p->window, 1 << 30); a.sinks = std::min(p->sinks, 1 << 30);      // caches have no more rows
  a.sl2 = (p->scale > 0.f ? p->scale : 1.0f / std::sqrt(static_cast<float>(p->head_dim))) * cd::kLog2e;
  a.out = out; a.lse = lse;
  hipStream_t st = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
#define CD_DISPATCH(T, D) return attend_impl<T, D>(p, a, max_cache_len, shared_table, shared_len, ws, st)
  if (p->dtype == CALIDROP_BF16) {
    if (p->head_dim == 128) CD_DISPATCH(cd::bf16_t, 128);
    CD_DISPATCH(cd::bf16_t, 64);
  }
  if (p->head_dim == 128) CD_DISPATCH(float, 128);
  CD_DISPATCH(float, 64);
#undef CD_DISPATCH
}

template <typename T, int D>
int launch_append(const cd::PagedAppendArgs& a, const calidrop_paged_params* p, dim3 grid, hipStream_t st) {
  if (p->rot_pairs == CALIDROP_ROT_HALVES) hipLaunchKernelGGL((cd::paged_append_kernel<T, D, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((cd::paged_append_kernel<T, D, false>), grid, dim3(256), 0, st, a);
  return launch_status("paged_append");
}

}  // namespace

extern "C" {

int calidrop_paged_append(const calidrop_paged_params* p, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                          const void* v, int64_t v_stride, const int32_t* new_offsets, int64_t total_new, int32_t max_new,
                          const int32_t* positions, const float* rot_table, int32_t n_positions, void* k_pages,
                          void* v_pages, const int32_t* page_table, const int32_t* cache_lens, int32_t* new_lens,
                          void* q_out, void* stream) {
  int rc;
  if ((rc = check_paged(p))) return rc;
  if (total_new < 0 || max_new < 1)
    return fail(CALIDROP_ESHAPE, "total_new >= 0 and max_new >= 1 expected (got %lld, %d)", static_cast<long long>(total_new), max_new);
  if (total_new > (int64_t{1} << 30)) return fail(CALIDROP_EUNSUPPORTED, "total_new exceeds 2^30");
  if (!new_offsets && total_new != p->batch)
    return fail(CALIDROP_ESHAPE, "without new_offsets every sequence has one token: total_new %lld is not the batch %d",
                static_cast<long long>(total_new), p->batch);
  if ((rc = check_ptrs({{cache_lens, "cache_lens"}, {new_lens, "new_lens"}}))) return rc;
  const int elem = p->dtype == CALIDROP_BF16 ? 2 : 4;
  if (total_new > 0) {
    if ((rc = check_ptrs({{k, "k"}, {v, "v"}, {k_pages, "k_pages"}, {v_pages, "v_pages"}, {page_table, "page_table"}}))) return rc;
    if (!q != !q_out) return fail(CALIDROP_EINVAL, "q and q_out go together");
    if (!aligned16(q) || !aligned16(q_out)) return fail(CALIDROP_EALIGN, "q or q_out is not 16-byte aligned");
    if (p->rot_dim) {
      if (!rot_table) return fail(CALIDROP_EINVAL, "rot_table is NULL although rot_dim is %d", p->rot_dim);
      if (n_positions < 1) return fail(CALIDROP_ESHAPE, "n_positions must be >= 1 (got %d)", n_positions);
      if (!aligned16(rot_table)) return fail(CALIDROP_EALIGN, "rot_table is not 16-byte aligned");
    }
    const struct { int64_t stride; int heads; const char* name; bool used; } strides[] = {
        {q_stride, p->n_q_heads, "q_stride", q != nullptr}, {k_stride, p->n_kv_heads, "k_stride", true}, {v_stride, p->n_kv_heads, "v_stride", true}};
    for (const auto& s : strides) {
      if (!s.used) continue;
      if (s.stride < static_cast<int64_t>(s.heads) * p->head_dim)
        return fail(CALIDROP_ESHAPE, "%s %lld is below the %d elements of a token", s.name, static_cast<long long>(s.stride), s.heads * p->head_dim);
      if (s.stride * elem % 16) return fail(CALIDROP_EALIGN, "%s %lld is no multiple of 16 bytes", s.name, static_cast<long long>(s.stride));
    }
    if (q && q == q_out && q_stride != static_cast<int64_t>(p->n_q_heads) * p->head_dim)
      return fail(CALIDROP_ESHAPE, "q can be rotated in place only where its tokens follow one another");
  }
  if (!aligned16(new_offsets) || !aligned16(positions)) return fail(CALIDROP_EALIGN, "new_offsets or positions is not 16-byte aligned");
  cd::PagedAppendArgs a{};
  a.q = static_cast<const char*>(q); a.k = static_cast<const char*>(k); a.v = static_cast<const char*>(v);
  a.q_stride = q_stride * elem; a.k_stride = k_stride * elem; a.v_stride = v_stride * elem;
  a.new_off = new_offsets; a.positions = positions; a.rot_table = rot_table;
  a.k_pages = static_cast<char*>(k_pages); a.v_pages = static_cast<char*>(v_pages); a.q_out = static_cast<char*>(q_out);
  a.lens = cache_lens; a.new_lens = new_lens;
  a.pages = pages_of(p, page_table, p->max_pages);
  a.total_new = total_new; a.batch = p->batch; a.Hq = p->n_q_heads; a.max_new = new_offsets ? max_new : 1;
  a.max_pages = p->max_pages; a.rot = p->rot_dim; a.n_positions = n_positions;
  a.tokens_per_group = a.max_new == 1 ? 1 : 4;
  const int groups = ceil_div(a.max_new, a.tokens_per_group);
  a.write_lens = groups == 1 || new_lens != cache_lens;
  const dim3 grid(groups, p->batch);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define CD_DISPATCH(T, D) rc = launch_append<T, D>(a, p, grid, st)
  if (p->dtype == CALIDROP_BF16) {
    if (p->head_dim == 128) CD_DISPATCH(cd::bf16_t, 128);
    else CD_DISPATCH(cd::bf16_t, 64);
  } else {
    if (p->head_dim == 128) CD_DISPATCH(float, 128);
    else CD_DISPATCH(float, 64);
  }
#undef CD_DISPATCH
  if (rc || a.write_lens) return rc;
  hipLaunchKernelGGL(cd::paged_lens_kernel, dim3(ceil_div(p->batch, 256)), dim3(256), 0, st, a);
  return launch_status("paged_lens");
}

size_t calidrop_paged_attend_workspace_bytes(const calidrop_paged_params* p, int64_t total_q, int32_t max_q_len, int32_t max_cache_len) {
  if (check_paged(p) != CALIDROP_OK || check_attend_sizes(p, total_q, max_q_len, max_cache_len) != CALIDROP_OK) return 0;
  return attend_bytes(p, total_q, max_q_len, max_cache_len);
}

int calidrop_paged_attend(const calidrop_paged_params* p, const void* q, const int32_t* q_offsets, int64_t total_q, int32_t max_q_len,
                          const void* k_pages, const void* v_pages, const int32_t* page_table, const int32_t* cache_lens,
                          int32_t max_cache_len, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check_paged(p))) return rc;
  if ((rc = check_attend_sizes(p, total_q, max_q_len, max_cache_len))) return rc;
  return attend_entry(p, q, q_offsets, total_q, max_q_len, k_pages, v_pages, nullptr, 0, page_table, cache_lens, max_cache_len, out, lse,
                      workspace, workspace_bytes, attend_bytes(p, total_q, max_q_len, max_cache_len), stream);
}

size_t calidrop_paged_attend_shared_workspace_bytes(const calidrop_paged_params* p, int64_t total_q, int32_t max_q_len,
                                                    int32_t max_cache_len, int32_t shared_len) {
  if (check_paged(p) != CALIDROP_OK || check_attend_sizes(p, total_q, max_q_len, max_cache_len) != CALIDROP_OK ||
      check_shared_sizes(p, shared_len) != CALIDROP_OK) return 0;
  return shared_bytes(p, total_q, max_q_len, max_cache_len, shared_len);
}

int calidrop_paged_attend_shared(const calidrop_paged_params* p, const void* q, const int32_t* q_offsets, int64_t total_q,
                                 int32_t max_q_len, const void* k_pages, const void* v_pages, const int32_t* shared_table,
                                 int32_t shared_len, const int32_t* page_table, const int32_t* cache_lens, int32_t max_cache_len,
                                 void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check_paged(p))) return rc;
  if ((rc = check_attend_sizes(p, total_q, max_q_len, max_cache_len))) return rc;
  if ((rc = check_shared_sizes(p, shared_len))) return rc;
  if (!shared_table) return fail(CALIDROP_EINVAL, "shared_table is NULL");
  return attend_entry(p, q, q_offsets, total_q, max_q_len, k_pages, v_pages, shared_table, shared_len, page_table, cache_lens,
                      max_cache_len, out, lse, workspace, workspace_bytes, shared_bytes(p, total_q, max_q_len, max_cache_len, shared_len),
                      stream);
}

}  // extern "C"
