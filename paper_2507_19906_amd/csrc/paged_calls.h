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
  if (static_cast<int64_t>(p->max_pages) * p->page_size > INT32_MAX)
    return fail(CALIDROP_EUNSUPPORTED, "max_pages * page_size exceeds 2^31 - 1 rows");
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

// magic = ceil(2^shift / d) with shift = 31 + ceil(log2 d); see cd::divide
cd::Divisor divisor(int d) {
  int bits = 0;
  while ((static_cast<int64_t>(1) << bits) < d) ++bits;
  const int shift = 31 + bits;
  return {static_cast<uint32_t>(((static_cast<uint64_t>(1) << shift) + d - 1) / d), shift};
}

cd::Pages pages_of(const calidrop_paged_params* p, const int32_t* table, int64_t stride) {
  cd::Pages pg{};
  pg.table = table; pg.table_stride = stride; pg.page_size = p->page_size; pg.n_pages = p->n_pages; pg.Hkv = p->n_kv_heads;
  pg.div = divisor(p->page_size);
  return pg;
}

// How an attention launch is cut up.  Up to 16 (token, head) rows stream the cache from memory to registers, more share tiles of
// it in LDS.
struct PagedPlan { bool stream; int rows, tile, least_shift; int64_t blocks, prefix, items, share, most_tiles; };      // share 0: a workgroup per block
// Workgroups that share the tiles of all KV heads: what the chip holds at a time of the bf16 kernels for D = 128.  Others fit in other
// numbers: of streams in fp32 with D = 128 512, in bf16 with D = 64 1024; of tiles in fp32 with D = 64 1280.  Streams measured with 512,
// 768 and 1024 (8 KV heads, us): fp32, D = 128, one sequence of 16000 rows 32.6, 41.7, 35.4, 4 of 8000 56.4, 65.0, 58.9, 32 of 1000 to
// 16000 404, 404, 395; bf16, D = 64, 4 of 16000 31.7, 31.0, 29.8, 16 of 8000 54.3, 51.4, 51.5; fp32, D = 64, 16 of 4000 55.1, 54.0,
// 59.2; bf16, D = 128: 512, 640 and 1024 no faster.  768 is within 8 % of the best but in fp32 with D = 128, where it costs up to 28 %.
constexpr int kPagedStreamPlaces = 768, kPagedTilePlaces = 512;
constexpr int64_t kPagedMostItems = 4096;                              // every workgroup adds up their tiles

// Most tiles that a block can need (cd::KeyTiles): under a window, the rows of the window and of the sinks can begin and end
// inside a tile each, and share one.
int64_t most_tiles(const calidrop_paged_params* p, int64_t q_len, int64_t max_len, int64_t rows, int64_t tile) {
  const int64_t all = (max_len + tile - 1) / tile;
  if (!p->window) return all;
  const int64_t tokens = std::min(q_len, rows / (p->n_q_heads / p->n_kv_heads) + 2);
  return std::min(all + 1, (p->window + tokens + tile - 1) / tile + 1 + (p->sinks + tile - 1) / tile);
}

// Blocks, and the workgroups that could share a KV head.  shared_len 0: no prefix.
PagedPlan paged_blocks(const calidrop_paged_params* p, int64_t total_q, int64_t q_len, int64_t max_len, int64_t shared_len) {
  PagedPlan plan{};
  const int64_t G = p->n_q_heads / p->n_kv_heads, rows = (shared_len ? std::max(total_q, q_len) : q_len) * G;
  const bool fp32 = p->dtype == CALIDROP_FP32;
  plan.stream = rows <= cd::kStreamRows;
  plan.rows = plan.stream ? cd::kStreamRows : fp32 ? cd::PagedTiles<float, 128>::kRows : cd::PagedTiles<cd::bf16_t, 128>::kRows;
  plan.tile = plan.stream || fp32 ? 32 : 64;
  plan.least_shift = 2;                                 // tiles of a share at least, setup included
  plan.blocks = (q_len * G + plan.rows - 1) / plan.rows;
  plan.prefix = shared_len ? (total_q * G + plan.rows - 1) / plan.rows : 0;
  plan.items = plan.prefix + p->batch * plan.blocks;
  plan.most_tiles = most_tiles(p, q_len, max_len, plan.rows, plan.tile);
  const int64_t most = std::max<int64_t>(1, (plan.stream ? kPagedStreamPlaces : kPagedTilePlaces) / p->n_kv_heads);
  const int setup = plan.stream ? cd::PagedBlock<16, 32>::kSetup : fp32 ? cd::PagedBlock<64, 32>::kSetup : cd::PagedBlock<128, 64>::kSetup;
  const int64_t tiles = std::min(plan.prefix, kPagedMostItems) * ((shared_len + plan.tile - 1) / plan.tile + setup) +
                        std::min(plan.items - plan.prefix, kPagedMostItems) * (plan.most_tiles + setup);
  plan.share = std::max<int64_t>(1, std::min(most, tiles >> plan.least_shift));
  return plan;
}

// A workgroup per block, or the tiles of a KV head shared evenly (and a launch that joins the parts): whichever is expected to take
// less time, from the longest cache the host knows of.  Measured in 191 calls (1 to 64 sequences, 1 to 4096 queries, caches of 100
// to 16512 rows, both types and head dimensions, 32 query and 8 KV heads), where the choice is 0.8 % behind the better form on average
// (21 % at most, one fp32 query of 300 rows); us a call, own block / shared:
//   streams of one query, bf16, D = 128: 1 sequence of 300 rows 9.1 / 11.9, of 600 13.3 / 11.9, of 4000 78 / 14; 16 of 600 17.7 /
//   20.1, of 1000 26.7 / 21.7, of 16000 364 / 174; 64 of 1000 46.6 / 55.3, of 4000 172 / 178.
//   tiles, bf16, D = 128: 64 queries at 1000 rows 29 / 24, at 16000 359 / 44; 512 queries of a prompt 17.6 / 32.5, at 8512 rows
//   193 / 102; 4 sequences of those 289 / 320; 2 prompts of 2048 87 / 170.
// The host does not know how the lengths of several sequences differ.  The shared form does not care (4 chunks of 300 to 512
// queries behind 8000 to 32000 rows 813 / 450, 64 queries of 1000 to 16000 rows 541 / 348), so it may cost `ragged` times the
// other there.  Calls of many blocks level themselves out.
struct PagedCost { float stream_tile, single, pair, pair_shared; };      // us a tile, alone on a compute unit and in pairs
PagedPlan plan_paged(const calidrop_paged_params* p, int64_t total_q, int64_t q_len, int64_t max_len, int64_t shared_len) {
  constexpr PagedCost kCost[2][2] = {{{.4f, 1.05f, 1.33f, 1.4f}, {.6f, 1.35f, 2.1f, 2.25f}}, {{.7f, 1.9f, 2.7f, 2.7f}, {1.2f, 3.f, 5.f, 5.f}}};
  const PagedCost& c = kCost[p->dtype == CALIDROP_FP32][p->head_dim == 128];
  PagedPlan plan = paged_blocks(p, total_q, q_len, max_len, shared_len);
  const int64_t tiles = plan.most_tiles, groups = plan.items * p->n_kv_heads;
  if (plan.share == 1 || plan.items > kPagedMostItems || plan.items * (8 + std::max(tiles, (shared_len + plan.tile - 1) / plan.tile)) >= (int64_t{1} << 31)) {
    plan.share = 0;
    return plan;
  }
  if (shared_len) return plan;                         // blocks of a long prefix and of short caches: never level
  if (groups >= 4 * kPagedTilePlaces) {
    plan.share = 0;
    return plan;
  }
  const float most = static_cast<float>(tiles), all = static_cast<float>(groups);
  float own, shared, ragged;
  if (plan.stream) {
    const float traffic = all * most * 64.f * static_cast<float>(p->head_dim) * (p->dtype == CALIDROP_FP32 ? 4.f : 2.f) / 6.1e6f;
    own = std::max(6.f + c.stream_tile * most, 3.f + traffic);
    shared = 12.f + traffic;
    ragged = 1.06f;
  } else {
    // the queries of a prompt see half of their own rows on average
    const float mean = p->window ? most : std::max(most - .5f * static_cast<float>(q_len) / static_cast<float>(plan.tile), .5f * most);
    const float places = kPagedTilePlaces, least = 2.f;
    const float parts = std::min(places, all * mean / least);
    // as many blocks as places: the long ones end alone
    own = 8.f + (groups <= kPagedTilePlaces / 2 ? c.single * most : groups <= kPagedTilePlaces ? c.pair * mean + c.single * (most - mean)
                                                                                            : std::max(c.single * most, c.pair * mean * all / places));
    shared = 14.f + 15.f * parts / places * static_cast<float>(plan.rows) / 128.f + c.pair_shared * std::max(mean * all / places, least);
    ragged = groups <= 2 * kPagedTilePlaces ? 1.15f : 1.f;
  }
  if (shared >= own * (p->batch > 1 ? ragged : 1.f)) plan.share = 0;
  return plan;
}

// The workspace: how blocks were cut, the parts, and with a prefix the whole blocks of both sides.
struct PagedRegions { size_t cut, part_ml, part_o, whole_ml, whole_o, total; };
PagedRegions paged_regions(const calidrop_paged_params* p, const PagedPlan& plan, int64_t total_q) {
  PagedRegions r{};
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
  const size_t parts = static_cast<size_t>(plan.share) * p->n_kv_heads * 2 * plan.rows, whole = plan.prefix ? static_cast<size_t>(total_q) * p->n_q_heads * 2 : 0;
  r.cut = take(static_cast<size_t>(std::min(plan.items, kPagedMostItems)) * sizeof(int4));
  r.part_ml = take(parts * sizeof(float2));
  r.part_o = take(parts * p->head_dim * sizeof(float));
  r.whole_ml = take(whole * sizeof(float2));
  r.whole_o = take(whole * p->head_dim * sizeof(float));
  r.total = std::max<size_t>(at, 256);
  return r;
}
size_t attend_bytes(const calidrop_paged_params* p, int64_t total_q, int64_t max_q_len, int64_t max_cache_len, int64_t shared_len) {
  return paged_regions(p, paged_blocks(p, total_q, max_q_len, max_cache_len, shared_len), total_q).total;
}

int check_attend_sizes(const calidrop_paged_params* p, int64_t total_q, int32_t max_q_len, int32_t max_cache_len) {
  if (total_q < 0 || max_q_len < 1 || max_cache_len < 0)
    return fail(CALIDROP_ESHAPE, "total_q >= 0, max_q_len >= 1 and max_cache_len >= 0 expected (got %lld, %d, %d)",
                static_cast<long long>(total_q), max_q_len, max_cache_len);
  if (total_q > (int64_t{1} << 29) / p->n_q_heads)
    return fail(CALIDROP_EUNSUPPORTED, "total_q * n_q_heads exceeds 2^29");
  const int64_t G = p->n_q_heads / p->n_kv_heads;
  if (max_q_len > (1 << 26) / G) return fail(CALIDROP_EUNSUPPORTED, "max_q_len * (n_q_heads / n_kv_heads) exceeds 2^26");
  if ((max_q_len * G + 63) / 64 * p->n_kv_heads * p->batch > 1 << 23)           // workgroups of 256 threads
    return fail(CALIDROP_EUNSUPPORTED, "batch * max_q_len * n_q_heads exceeds 2^29");
  if (max_cache_len > paged_capacity(p))
    return fail(CALIDROP_ESHAPE, "max_cache_len %d exceeds the max_pages * page_size = %lld rows of a table", max_cache_len,
                static_cast<long long>(paged_capacity(p)));
  if (max_cache_len > (1 << 30)) return fail(CALIDROP_EUNSUPPORTED, "max_cache_len %d exceeds 2^30", max_cache_len);
  return CALIDROP_OK;
}
// No sequence has more tokens than the call, whatever the host's bound says.
int64_t most_tokens(int64_t total_q, int64_t max_q_len) { return std::min(max_q_len, std::max<int64_t>(total_q, 1)); }

// After check_attend_sizes.  A prefix adds as many blocks again to the first launch, and its second has four rows to a workgroup;
// a launch holds fewer than 2^32 threads in a direction, 2^24 workgroups of 256.
int check_shared_sizes(const calidrop_paged_params* p, int64_t total_q, int32_t max_q_len, int32_t shared_len) {
  if (shared_len < 1) return fail(CALIDROP_ESHAPE, "shared_len must be >= 1 (got %d)", shared_len);
  if (shared_len > (1 << 30)) return fail(CALIDROP_EUNSUPPORTED, "shared_len %d exceeds 2^30", shared_len);
  if (p->window || p->sinks) return fail(CALIDROP_EUNSUPPORTED, "a shared prefix goes without window and sinks (got %d, %d)", p->window, p->sinks);
  const int64_t q_len = most_tokens(total_q, max_q_len), rows = q_len * (p->n_q_heads / p->n_kv_heads);
  if (paged_blocks(p, total_q, q_len, 0, shared_len).items * p->n_kv_heads >= 1 << 24)
    return fail(CALIDROP_EUNSUPPORTED, "the prefix and the sequences together reach 2^24 blocks of queries");
  if ((rows + 3) / 4 >= 1 << 24)
    return fail(CALIDROP_EUNSUPPORTED, "with a prefix, max_q_len * (n_q_heads / n_kv_heads) exceeds 2^26 - 4");
  return CALIDROP_OK;
}

template <typename T, int D>
int attend_impl(const calidrop_paged_params* p, cd::PagedAttendArgs& a, char* ws, hipStream_t st) {
  const PagedPlan plan = plan_paged(p, a.total_q, a.max_q_len, a.max_len, a.shared_len);
  const PagedRegions R = paged_regions(p, plan, a.total_q);
  a.blocks = static_cast<int>(plan.blocks); a.items = static_cast<int>(plan.items); a.prefix_items = static_cast<int>(plan.prefix);
  a.share = static_cast<int>(plan.share);
  a.least_shift = plan.least_shift;
  a.by_blocks = divisor(a.blocks); a.by_G = divisor(a.G); a.by_Hkv = divisor(p->n_kv_heads);
  a.cut = reinterpret_cast<int4*>(ws + R.cut);
  a.part_ml = reinterpret_cast<float2*>(ws + R.part_ml); a.part_o = reinterpret_cast<float*>(ws + R.part_o);
  a.whole_ml = reinterpret_cast<float2*>(ws + R.whole_ml); a.whole_o = reinterpret_cast<float*>(ws + R.whole_o);
  void (*kernel)(cd::PagedAttendArgs);
  // Behind a prefix the few queries of a sequence's own rows go through the tile kernel too, a wave of four at work: streamed
  // without LDS in the same launch, as the streaming kernel does alone, they were no faster (64 queries, 32768 + 0 to 512 rows
  // 72 for 67 us; 256 queries, 8000 + 10 to 300 rows 86 both), since two waves on a SIMD hide less than loads two tiles ahead.
  if (plan.stream) kernel = plan.share ? cd::paged_stream_kernel<T, D, true> : cd::paged_stream_kernel<T, D, false>;
  else if constexpr (sizeof(T) == 2) kernel = plan.share ? cd::paged_tile_kernel<D, true> : cd::paged_tile_kernel<D, false>;
  else kernel = plan.share ? cd::paged_tile32_kernel<D, true> : cd::paged_tile32_kernel<D, false>;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>((plan.share ? plan.share : plan.items) * p->n_kv_heads)), dim3(256), 0, st, a);
  const int rc = launch_status("paged_attend");
  if (rc || (!plan.prefix && !plan.share)) return rc;
  cd::PagedJoinArgs j{a, plan.rows};
  const int64_t rows = static_cast<int64_t>(a.max_q_len) * a.G;
  const unsigned Hkv = p->n_kv_heads, nb = p->batch;
  if (rows * Hkv * nb >= 4096) hipLaunchKernelGGL((cd::paged_join_kernel<T, D, 1>), dim3(static_cast<unsigned>((rows + 3) / 4), Hkv, nb), dim3(256), 0, st, j);
  else if (rows * Hkv * nb > 256) hipLaunchKernelGGL((cd::paged_join_kernel<T, D, 4>), dim3(static_cast<unsigned>(rows), Hkv, nb), dim3(256), 0, st, j);
  else hipLaunchKernelGGL((cd::paged_join_kernel<T, D, 16>), dim3(static_cast<unsigned>(rows), Hkv, nb), dim3(1024), 0, st, j);
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
  a.shared_table = shared_table; a.shared_len = shared_len;
  a.total_q = total_q; a.batch = p->batch; a.Hq = p->n_q_heads; a.G = p->n_q_heads / p->n_kv_heads;
  a.max_q_len = q_offsets ? static_cast<int>(most_tokens(total_q, max_q_len)) : 1;
  a.window = std::min(p->window, 1 << 30); a.sinks = std::min(p->sinks, 1 << 30);      // caches have no more rows
  a.sl2 = (p->scale > 0.f ? p->scale : 1.0f / std::sqrt(static_cast<float>(p->head_dim))) * cd::kLog2e;
  a.out = out; a.lse = lse;
  hipStream_t st = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
#define CD_DISPATCH(T, D) return attend_impl<T, D>(p, a, ws, st)
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
  if (total_new > (int64_t{1} << 30) || max_new > (1 << 25)) return fail(CALIDROP_EUNSUPPORTED, "total_new exceeds 2^30 or max_new 2^25");
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
  a.units = (p->rot_pairs == CALIDROP_ROT_HALVES ? p->head_dim - p->rot_dim / 2 : p->head_dim) * elem / 16;
  a.by_units = divisor(a.units);
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
  return attend_bytes(p, total_q, max_q_len, max_cache_len, 0);
}

int calidrop_paged_attend(const calidrop_paged_params* p, const void* q, const int32_t* q_offsets, int64_t total_q, int32_t max_q_len,
                          const void* k_pages, const void* v_pages, const int32_t* page_table, const int32_t* cache_lens,
                          int32_t max_cache_len, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check_paged(p))) return rc;
  if ((rc = check_attend_sizes(p, total_q, max_q_len, max_cache_len))) return rc;
  return attend_entry(p, q, q_offsets, total_q, max_q_len, k_pages, v_pages, nullptr, 0, page_table, cache_lens, max_cache_len, out, lse,
                      workspace, workspace_bytes, attend_bytes(p, total_q, max_q_len, max_cache_len, 0), stream);
}

size_t calidrop_paged_attend_shared_workspace_bytes(const calidrop_paged_params* p, int64_t total_q, int32_t max_q_len,
                                                    int32_t max_cache_len, int32_t shared_len) {
  if (check_paged(p) != CALIDROP_OK || check_attend_sizes(p, total_q, max_q_len, max_cache_len) != CALIDROP_OK ||
      check_shared_sizes(p, total_q, max_q_len, shared_len) != CALIDROP_OK) return 0;
  return attend_bytes(p, total_q, max_q_len, max_cache_len, shared_len);
}

int calidrop_paged_attend_shared(const calidrop_paged_params* p, const void* q, const int32_t* q_offsets, int64_t total_q,
                                 int32_t max_q_len, const void* k_pages, const void* v_pages, const int32_t* shared_table,
                                 int32_t shared_len, const int32_t* page_table, const int32_t* cache_lens, int32_t max_cache_len,
                                 void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check_paged(p))) return rc;
  if ((rc = check_attend_sizes(p, total_q, max_q_len, max_cache_len))) return rc;
  if ((rc = check_shared_sizes(p, total_q, max_q_len, shared_len))) return rc;
  if (!shared_table) return fail(CALIDROP_EINVAL, "shared_table is NULL");
  return attend_entry(p, q, q_offsets, total_q, max_q_len, k_pages, v_pages, shared_table, shared_len, page_table, cache_lens,
                      max_cache_len, out, lse, workspace, workspace_bytes, attend_bytes(p, total_q, max_q_len, max_cache_len, shared_len),
                      stream);
}

}  // extern "C"
