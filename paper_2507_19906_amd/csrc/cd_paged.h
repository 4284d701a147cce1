// Keys and values in pages: appending new rows (with the position rotation applied on the way) and attention that reads
// them - prompts, chunks of prompts and single tokens, whole contexts or a sliding window with a few first tokens that stay
// visible, with or without a prefix that all sequences share.
//
// A page holds page_size rows of every KV head, [Hkv][page_size][D]: the layout of a prompt or compressed cache of that many
// rows.  Row r of sequence b is row r % page_size of page table[b][r / page_size].
#pragma once
#include "cd_common.h"
#include "cd_score.h"

namespace cd {

// ---- where a row is ---------------------------------------------------------------------------------------------------

// x / d for 0 <= x < 2^31 as one 64-bit product and shift: magic = ceil(2^shift / d), shift = 31 + ceil(log2 d).  magic < 2^32
// and x * (magic * d - 2^shift) < 2^31 * d <= 2^shift, so the quotient is exact.
struct Divisor { uint32_t magic; int shift; };
__device__ __forceinline__ int divide(int x, Divisor d) {
  return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(x)) * d.magic) >> d.shift);
}

struct Pages {
  const int32_t* table;      // entries of sequence b at table + b * table_stride
  int64_t table_stride;
  int page_size, n_pages, Hkv;
  Divisor div;               // by page_size
};

// Row `pos` of KV head g as a row number of the page buffers (rows of D elements; below 2^32 for every buffer that fits the
// card).  An entry that names no page is read as the nearest one that exists.
__device__ __forceinline__ uint32_t page_row(const Pages& pg, const int32_t* table, int g, int pos) {
  const int e = divide(pos, pg.div);
  const int page = min(max(table[e], 0), pg.n_pages - 1);
  return (static_cast<uint32_t>(page) * pg.Hkv + g) * pg.page_size + (pos - e * pg.page_size);
}

// ---- append -------------------------------------------------------------------------------------------------------------

struct PagedAppendArgs {
  const char* q; const char* k; const char* v;      // [total][heads][D], tokens q_stride / k_stride / v_stride bytes apart
  int64_t q_stride, k_stride, v_stride;
  const int32_t* new_off;                           // [batch+1] tokens of a sequence, or NULL: one each
  const int32_t* positions;                         // [total] place in the text, or NULL: the row in the cache
  const float* rot_table;                           // [n_positions][rot]: cosines, then sines
  char* k_pages; char* v_pages; char* q_out;
  const int32_t* lens; int32_t* new_lens;
  Pages pages;
  int64_t total_new;
  int batch, Hq, max_new, max_pages, rot, n_positions, tokens_per_group, write_lens;
  int units;                                        // of a turned head: pieces of 16 bytes, or pairs of them and single ones
  Divisor by_units;
};

// 16 bytes of a row as 32-bit floats, and back.
template <typename T> __device__ __forceinline__ void unpack16(const u32x4& x, float (&f)[Elem<T>::kPer16B]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t u = x[e];
    if constexpr (sizeof(T) == 2) {
      f[2 * e] = as_f32(u << 16);
      f[2 * e + 1] = as_f32(u & 0xffff0000u);
    } else {
      f[e] = as_f32(u);
    }
  }
}
template <typename T> __device__ __forceinline__ u32x4 pack16(const float (&f)[Elem<T>::kPer16B]) {
  u32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) x[e] = pack_bf16x2(f[2 * e], f[2 * e + 1]);
    else x[e] = __builtin_bit_cast(uint32_t, f[e]);
  }
  return x;
}
template <int N> __device__ __forceinline__ void load_floats(const float* p, float (&f)[N]) {
  typedef float vec __attribute__((ext_vector_type(N < 4 ? N : 4)));
  constexpr int V = N < 4 ? N : 4;
#pragma unroll
  for (int e = 0; e < N; e += V) {
    const vec x = *reinterpret_cast<const vec*>(p + e);
#pragma unroll
    for (int y = 0; y < V; ++y) f[e + y] = x[y];
  }
}

// A workgroup takes tokens_per_group tokens of one sequence, its four waves one token together or one each; a lane 16 bytes of one
// head (two pieces of 16 bytes, the two elements of its pairs, where those lie half the rotated part apart).  What belongs to a
// token - its page, its position - is the same in every lane.  The rotation is in 32 bits, rounded once to the storage type.
// Bound by the bytes of the heads, read and written once.
template <typename T, int D, bool kHalves>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int E = Elem<T>::kPer16B, kChunks = D / E;
  constexpr int64_t kRow = D * sizeof(T);
  const int b = blockIdx.y;
  int64_t t0 = b, t1 = b + 1;
  if (a.new_off) { t0 = a.new_off[b]; t1 = a.new_off[b + 1]; }
  t0 = min(max(t0, static_cast<int64_t>(0)), a.total_new);
  t1 = min(max(t1, t0), a.total_new);
  const int n = static_cast<int>(min(t1 - t0, static_cast<int64_t>(a.max_new)));
  const int len = a.lens[b];
  const bool fits = len >= 0 && static_cast<int64_t>(len) + n <= static_cast<int64_t>(a.max_pages) * a.pages.page_size;
  __syncthreads();                                  // everyone has read the length before it changes
  if (a.write_lens && blockIdx.x == 0 && threadIdx.x == 0) a.new_lens[b] = fits ? len + n : len;
  const int wave = wave_index(), lane = threadIdx.x & 63;
  const bool together = a.tokens_per_group == 1;
  const int t = static_cast<int>(blockIdx.x) * a.tokens_per_group + (together ? 0 : wave);
  if (t >= n) return;
  const int64_t token = t0 + t;
  const int at = len + t, rot = a.rot, Hkv = a.pages.Hkv;
  const int first = together ? 64 * wave + lane : lane, step = together ? 256 : 64;
  const int e = fits ? divide(at, a.pages.div) : 0;
  const int page = fits ? a.pages.table[b * a.pages.table_stride + e] : -1;
  const bool stored = page >= 0 && page < a.pages.n_pages;
  const int64_t slot = stored ? (static_cast<int64_t>(page) * Hkv * a.pages.page_size + (at - e * a.pages.page_size)) * kRow : 0;
  const int64_t head = a.pages.page_size * kRow;    // from one KV head of a page to the next
  const float* cs = a.rot_table;
  if (rot) cs += static_cast<int64_t>(min(max(a.positions ? a.positions[token] : at, 0), a.n_positions - 1)) * rot;
  const int turned = (kHalves ? rot / 2 : rot) / E;                    // units that turn: a pair of pieces, or a piece
  auto turn_heads = [&](const char* src, char* dst, int64_t dst_head, int heads) {
    for (int item = first; item < heads * a.units; item += step) {
      const int h = divide(item, a.by_units);
      int u = item - h * a.units;
      const char* x_at = src + h * kRow;
      char* to = dst + h * dst_head;
      if (u >= turned) {
        if (kHalves) u += turned;                                      // the pieces behind the pairs
        st16(to + u * 16, ld16_stream(x_at + u * 16));
      } else if constexpr (kHalves) {
        const int far = turned * 16;
        float x[E], y[E], c[E], s[E], p[E], q[E];
        const u32x4 xb = ld16_stream(x_at + u * 16), yb = ld16_stream(x_at + u * 16 + far);
        load_floats(cs + u * E, c);
        load_floats(cs + rot / 2 + u * E, s);
        unpack16<T>(xb, x);
        unpack16<T>(yb, y);
#pragma unroll
        for (int i = 0; i < E; ++i) { p[i] = x[i] * c[i] - y[i] * s[i]; q[i] = y[i] * c[i] + x[i] * s[i]; }
        st16(to + u * 16, pack16<T>(p));
        st16(to + u * 16 + far, pack16<T>(q));
      } else {
        float x[E], c[E / 2], s[E / 2], p[E];
        const u32x4 xb = ld16_stream(x_at + u * 16);
        load_floats(cs + u * (E / 2), c);
        load_floats(cs + rot / 2 + u * (E / 2), s);
        unpack16<T>(xb, x);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          p[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * s[i];
          p[2 * i + 1] = x[2 * i + 1] * c[i] + x[2 * i] * s[i];
        }
        st16(to + u * 16, pack16<T>(p));
      }
    }
  };
  if (a.q) turn_heads(a.q + token * a.q_stride, a.q_out + token * a.Hq * kRow, kRow, a.Hq);
  if (!stored) return;
  turn_heads(a.k + token * a.k_stride, a.k_pages + slot, head, Hkv);
  const char* v = a.v + token * a.v_stride;
  for (int item = first; item < Hkv * kChunks; item += step)
    st16(a.v_pages + slot + item / kChunks * head + item % kChunks * 16, ld16_stream(v + item * 16));
}

// new_lens of calls whose sequences have several workgroups, where it is the array the lengths are read from.
__global__ __launch_bounds__(256) void paged_lens_kernel(PagedAppendArgs a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= a.batch) return;
  int64_t t0 = min(max(static_cast<int64_t>(a.new_off[b]), static_cast<int64_t>(0)), a.total_new);
  int64_t t1 = min(max(static_cast<int64_t>(a.new_off[b + 1]), t0), a.total_new);
  const int n = static_cast<int>(min(t1 - t0, static_cast<int64_t>(a.max_new)));
  const int len = a.lens[b];
  const bool fits = len >= 0 && static_cast<int64_t>(len) + n <= static_cast<int64_t>(a.max_pages) * a.pages.page_size;
  a.new_lens[b] = fits ? len + n : len;
}

// ---- attention ------------------------------------------------------------------------------------------------------------
//
// The work of a call is made of blocks: the queries of one sequence and KV head, as (token, head of the group) rows, cut into
// blocks of kRows rows.  A block needs the tiles of its cache that one of its queries sees.  Either every workgroup has a block,
// or, where there are too few blocks or their caches differ too much, a fixed number of workgroups shares the tiles of all
// blocks of a KV head evenly, in order: a workgroup's share may begin and end inside a block.  The lengths are known to the
// device alone, so each workgroup adds them up for itself.  Results of parts of blocks go to the workspace and are joined by a
// second launch.  A prefix that all sequences share is one more sequence, ahead of the others, whose queries are those of the
// whole call and see every row; a (token, head) then has two blocks, whose results are joined.

struct PagedAttendArgs {
  const void* q;             // [total_q][Hq][D]
  const int32_t* q_off;      // [batch+1], or NULL: one token each
  const void* k; const void* v;
  const int32_t* lens;       // rows of each sequence's cache
  Pages pages;
  const int32_t* shared_table;
  int shared_len, max_len;
  int64_t total_q;
  int batch, Hq, G, max_q_len;
  Divisor by_G, by_blocks, by_Hkv;
  int window, sinks;         // window 0: no limit
  float sl2;                 // scale * log2(e)
  void* out; float* lse;
  int blocks, items;         // blocks of a sequence at most, of all sequences and the prefix
  int prefix_items;          // those of the prefix come first; their results are kept apart
  int share;                 // workgroups that share the tiles of a KV head, 0: one per block
  int least_shift;           // a share has 2^least_shift tiles at least
  int4* cut;                 // [items] how a block was cut: first and last workgroup, 1 if it is not the first one's first
  float* part_o;             // [Hkv][share][2][kRows][D] the parts of the block a workgroup begins with, and of the one it ends with
  float2* part_ml;           // [Hkv][share][2][kRows]    unnormalised outputs; (maximum in log2 units, sum)
  float* whole_o;            // with a prefix whole blocks go to the workspace too: [2][total_q][Hq][D], the prefix's second
  float2* whole_ml;          // [2][total_q][Hq]
};

// The tokens of sequence b: first token and number.
__device__ __forceinline__ int query_range(const PagedAttendArgs& a, int b, int64_t& q0) {
  int64_t q1;
  if (a.q_off) { q0 = a.q_off[b]; q1 = a.q_off[b + 1]; } else { q0 = b; q1 = b + 1; }
  q0 = min(max(q0, static_cast<int64_t>(0)), a.total_q);
  q1 = min(max(q1, q0), a.total_q);
  return static_cast<int>(min(q1 - q0, static_cast<int64_t>(a.max_q_len)));
}
// The tiles of TK rows that a block of queries needs: those that hold one of the first `sinks` rows, then those from the
// oldest query's window to the newest query.  A tile takes part with the rows of its range only, so that a tile of both
// ranges counts no row twice, and rows outside (freed pages, rows behind the end) are never read.
template <int TK>
struct KeyTiles {
  int n_sink, n, first, sink_end, lo, hi;
  __device__ __forceinline__ void init(int len, int pos_min, int pos_max, int window, int sinks) {
    hi = min(len, pos_max + 1);
    lo = window ? max(0, pos_min - window + 1) : 0;
    sink_end = window ? min(sinks, hi) : 0;
    if (lo <= sink_end) { lo = 0; sink_end = 0; }      // one range
    n_sink = (sink_end + TK - 1) / TK;
    first = lo / TK;
    n = hi > 0 ? n_sink + (hi + TK - 1) / TK - first : 0;
  }
  __device__ __forceinline__ void tile(int u, int& base, int& from, int& to) const {
    const bool s = u < n_sink;
    base = (s ? u : first + u - n_sink) * TK;
    from = s ? 0 : lo;
    to = s ? sink_end : hi;
  }
};

// kSetup: tiles in whose time a workgroup gets ready for a block and hands over its results.  They count as tiles ahead of its own,
// which a block's first workgroup has.  (Streams; fp32 and bf16 tiles.  None: 81 us for 64 queries behind a prefix of 32768 rows
// that take 67 so, 33 for 20 for fp32 prompts of 65 to 512 tokens.)
template <int kRows, int TK>
struct PagedBlock {
  static constexpr int kSetup = kRows == 16 ? 4 : kRows == 64 ? 3 : 2;
  int R, r0, len, past;      // past: row of the first query, len in a prefix
  bool prefix;
  int64_t q0;                // first token
  const int32_t* table;
  KeyTiles<TK> kt;
  __device__ __forceinline__ void init(const PagedAttendArgs& a, int item) {
    prefix = item < a.prefix_items;
    if (prefix) {
      r0 = item * kRows;
      q0 = 0;
      R = static_cast<int>(a.total_q) * a.G;
      past = len = a.shared_len;
      table = a.shared_table;
    } else {
      item -= a.prefix_items;
      const int b = divide(item, a.by_blocks);
      r0 = (item - b * a.blocks) * kRows;
      const int nq = query_range(a, b, q0);
      R = nq * a.G;
      len = min(max(a.lens[b], 0), a.max_len);
      past = len - nq;
      table = a.pages.table + b * a.pages.table_stride;
    }
    kt.init(len, pos_of(a, r0), pos_of(a, min(r0 + kRows, R) - 1), a.window, a.sinks);
  }
  // the last row that block row r sees
  __device__ __forceinline__ int pos_of(const PagedAttendArgs& a, int r) const { return past + divide(r, a.by_G); }
  // tiles with those of the setup, 0 where there is no such block
  __device__ __forceinline__ int weight() const { return r0 < R ? kt.n + kSetup : 0; }
};

// The tiles lo .. hi-1 of all blocks of KV head g are workgroup w's; they begin in block `item`, whose first tile is `start`.
struct PagedShare { int lo, hi, start, item, g, w; };      // tiles of a launch: below 2^31

template <int kRows, int TK, bool kShare>
__device__ __forceinline__ PagedShare paged_share(const PagedAttendArgs& a, uint32_t* scratch) {
  PagedShare s;
  const int Hkv = a.pages.Hkv, x = blockIdx.x;
  PagedBlock<kRows, TK> blk;
  s.lo = s.hi = s.start = s.item = s.w = 0;
  if constexpr (!kShare) {
    // blocks of a (sequence, KV head) behind one L2 and the heads of every sequence spread over the XCDs, which workgroups go
    // to in turn; the longest blocks of a prompt first
    const int heads = Hkv * a.batch;
    int rb, gb;
    if (a.prefix_items) { gb = x % Hkv; rb = a.blocks - 1 - x / Hkv; }
    else {
      const int slot = heads % 8 == 0 ? x / 8 : x, gs = divide(slot, a.by_blocks);
      rb = slot - gs * a.blocks;
      gb = heads % 8 == 0 ? gs * 8 + x % 8 : gs;
    }
    const int b = divide(gb, a.by_Hkv);
    s.g = gb - b * Hkv;
    s.item = b * a.blocks + (a.blocks - 1 - rb);
    return s;
  }
  // the tiles of all blocks added up: a thread has up to (items + 255) / 256 blocks in a row
  const int tid = threadIdx.x, per = (a.items + 255) / 256, i0 = tid * per, i1 = min(i0 + per, a.items);
  uint32_t mine = 0, before = 0;
  int total;
  if (a.items == 1) {
    blk.init(a, 0);
    total = blk.weight();
  } else {
    for (int it = i0; it < i1; ++it) { blk.init(a, it); mine += blk.weight(); }
    const uint32_t upto = wave_inclusive_scan(mine);
    if ((tid & 63) == 63) scratch[tid >> 6] = upto;
    __syncthreads();
    const uint32_t t0 = scratch[0], t1 = scratch[1], t2 = scratch[2], t3 = scratch[3];
    before = upto - mine + (tid >= 64 ? t0 : 0) + (tid >= 128 ? t1 : 0) + (tid >= 192 ? t2 : 0);
    total = __builtin_amdgcn_readfirstlane(t0 + t1 + t2 + t3);
  }
  const int W = min(max(total >> a.least_shift, 1), a.share);
  if (W == a.share && 8 % Hkv == 0 && a.share % (8 / Hkv) == 0) {      // neighbouring shares behind one L2
    const int xcd = x % 8;
    s.g = xcd % Hkv;
    s.w = xcd / Hkv * (a.share / (8 / Hkv)) + x / 8;
  } else {
    s.w = divide(x, a.by_Hkv);
    s.g = x - s.w * Hkv;
  }
  if (s.w >= W) return s;
  const int each = static_cast<uint32_t>(total) / static_cast<uint32_t>(W), more = total - each * W;      // the first `more` have one tile more
  s.lo = each * s.w + min(s.w, more);
  s.hi = s.lo + each + (s.w < more ? 1 : 0);
  if (a.items > 1) {
    if (before <= static_cast<uint32_t>(s.lo) && static_cast<uint32_t>(s.lo) < before + mine) {
      uint32_t at = before;
      int it = i0;
      if (per > 1)
        for (; it < i1; ++it) {
          blk.init(a, it);
          if (static_cast<uint32_t>(s.lo) < at + static_cast<uint32_t>(blk.weight())) break;
          at += blk.weight();
        }
      scratch[4] = it;
      scratch[5] = at;
    }
    __syncthreads();
    s.item = __builtin_amdgcn_readfirstlane(scratch[4]);
    s.start = __builtin_amdgcn_readfirstlane(scratch[5]);
    __syncthreads();
  }
  return s;
}

// Where the results of workgroup rows go: out and lse, the whole rows' partials, or a part's.
struct PagedTarget {
  bool final_rows, by_row;
  float* o; float2* ml;
};
// `begins`: the block is the first of the workgroup's.
template <int kRows, int D, bool kShare, int TK>
__device__ __forceinline__ PagedTarget paged_target(const PagedAttendArgs& a, const PagedShare& s, const PagedBlock<kRows, TK>& blk, int u0, int u1,
                                                    bool begins) {
  const int64_t side = blk.prefix ? a.total_q * a.Hq : 0;
  const PagedTarget whole{a.prefix_items == 0, true, a.whole_o + side * D, a.whole_ml + side};
  if constexpr (!kShare) return whole;
  if (s.g == 0 && threadIdx.x == 0) {                  // the heads are cut alike
    int* cut = reinterpret_cast<int*>(a.cut + s.item);
    if (u0 == 0) { cut[0] = s.w; cut[2] = begins ? 0 : 1; }
    if (u1 == blk.kt.n) cut[1] = s.w;
  }
  if (u0 == 0 && u1 == blk.kt.n) return whole;
  const int64_t slot = (static_cast<int64_t>(s.g) * a.share + s.w) * 2 + (begins ? 0 : 1);
  return PagedTarget{false, false, a.part_o + slot * kRows * D, a.part_ml + slot * kRows};
}

// f(block, u0, u1, first of the share) for every block that the workgroup has tiles u0 .. u1-1 of.
template <int kRows, int TK, bool kShare, typename F>
__device__ __forceinline__ void paged_blocks(const PagedAttendArgs& a, PagedShare& s, F&& f) {
  PagedBlock<kRows, TK> blk;
  if constexpr (!kShare) {
    blk.init(a, s.item);
    if (blk.r0 < blk.R) f(blk, 0, blk.kt.n, true);
    return;
  }
  bool begins = true;
  while (s.lo < s.hi) {
    blk.init(a, s.item);
    const int n = blk.weight();
    if (n > 0) {
      // a share that ends within the setup leaves the block to the next, one that begins there has it from its first tile on
      const int u0 = max(s.lo - s.start - blk.kSetup, 0), u1 = min(n, s.hi - s.start) - blk.kSetup;
      if (u1 > 0 || (u1 == 0 && blk.kt.n == 0)) {
        f(blk, u0, u1, begins);
        begins = false;
      }
    }
    s.start += n;
    s.lo = s.start;
    ++s.item;
  }
}

// A wave with 16 (token, head) rows, in the layout of the 16 x 16 products (lane l = 16 c + i).  S^T = K Q^T puts a query into a
// column, so that its softmax weights stay in the lanes that made them and are the B operand of O^T += V^T P^T as they are: the
// rows of a tile are dealt to the K operand in the order in which the products want the weights.
template <typename T, int D>
struct PagedWave {
  static constexpr int EPL = Elem<T>::kPer16B, KD = Elem<T>::kStepK, NK = D / KD;
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int NP = kBf16 ? 1 : D / 64;            // 16-byte pieces of a V row per lane (bf16, D = 64: 8 bytes)
  static constexpr int NX = kBf16 ? D / 16 : 4;            // elements of a piece
  static constexpr int NACC = NP * NX;                     // O^T tiles: 16 rows (slots of D) x 16 queries
  typedef uint32_t VPiece __attribute__((ext_vector_type(kBf16 && D == 64 ? 2 : 4)));

  u32x4 qf[NK];
  f32x4 o[NACC];
  float m, l;                                      // running maximum (log2 units) and this lane's share of the sum

  // row of a tile that lane (i, c) loads for K group t, and for slot e of V
  static __device__ __forceinline__ int k_row(int t, int i) { return kBf16 ? 8 * (i >> 2) + 4 * t + (i & 3) : 16 * t + i; }
  static __device__ __forceinline__ int v_row(int e, int c) { return kBf16 ? 8 * c + e : 16 * (e >> 2) + 4 * c + (e & 3); }
  // row of a tile of weight r of K group t in lane group c
  static __device__ __forceinline__ int p_row(int t, int c, int r) { return kBf16 ? 8 * c + 4 * t + r : 16 * t + 4 * c + r; }
  // first of the elements of D that lane group c holds of output piece p: o[p NX + x][r] is element d_first + r NX + x
  static __device__ __forceinline__ int d_first(int p, int c) { return p * 64 + c * 4 * NX; }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int x = 0; x < NACC; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void load_q(const T* q, bool valid, int c) {
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) qf[kk] = valid ? ld16(q + kk * KD + c * EPL) : zero16();
  }
  // Logits to weights: s[x] are those of K group t0 + x of the tile at `base`; sums and outputs so far are rescaled to the new
  // maximum.
  template <int N>
  __device__ __forceinline__ void weigh(f32x4* s, int t0, int base, int from, int to, int pos, const PagedAttendArgs& a, int c) {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = base + p_row(t0 + t, c, r);
        const bool see = j >= from && j < to && j <= pos && (a.window == 0 || j > pos - a.window || j < a.sinks);
        s[t][r] = see ? s[t][r] * a.sl2 : -INFINITY;
        top = fmaxf(top, s[t][r]);
      }
    const float mn = fmaxf(m, col4_max(top));
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float f = mn == m ? 1.f : fast_exp2(m - ref);
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) { s[t][r] = fast_exp2(s[t][r] - ref); sum += s[t][r]; }
    l = l * f + sum;
    if (__any(f != 1.f)) {
#pragma unroll
      for (int x = 0; x < NACC; ++x) o[x] *= f;
    }
  }
  // The results of this lane's column, block row `br`, (token, head) row `row`; l is the whole sum.
  __device__ __forceinline__ void write(const PagedTarget& to, const PagedAttendArgs& a, int64_t row, int br, int c) const {
    if (to.final_rows) {
      const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int x = 0; x < NX; ++x)
            store_elem(static_cast<T*>(a.out), row * D + d_first(p, c) + r * NX + x, o[p * NX + x][r] * inv);
      if (c == 0) a.lse[row] = l > 0.f ? (m + fast_log2(l)) * kLn2 : -INFINITY;
      return;
    }
    const int64_t at = to.by_row ? row : br;
    if (c == 0) to.ml[at] = float2{m, l};
    if (l == 0.f) return;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 0; x < NX; x += 4)
          *reinterpret_cast<f32x4*>(to.o + at * D + d_first(p, c) + r * NX + x) =
              f32x4{o[p * NX + x][r], o[p * NX + x + 1][r], o[p * NX + x + 2][r], o[p * NX + x + 3][r]};
  }

  __device__ __forceinline__ void load_k(const T* k, uint32_t rid, int i, int c, u32x4 (&kf)[2][NK]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const T* kp = k + static_cast<int64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(rid), k_row(t, i)))) * D + c * EPL;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) kf[t][kk] = ld16_stream(kp + kk * KD);
    }
  }
  __device__ __forceinline__ void load_v(const T* v, uint32_t rid, int i, int c, VPiece (&vf)[8][NP]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const T* vp = v + static_cast<int64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(rid), v_row(e, c)))) * D + i * NX;
#pragma unroll
      for (int p = 0; p < NP; ++p) vf[e][p] = __builtin_nontemporal_load(reinterpret_cast<const VPiece*>(vp + p * 64));
    }
  }
  // A operand of output tile (p, x): slot i holds element p 64 + i NX + x of the rows of lane group c
  __device__ __forceinline__ u32x4 v_operand(const VPiece (&vf)[8][NP], int p, int x, int t) const {
    u32x4 f;
    if constexpr (kBf16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = vf[2 * j][0][x >> 1], hi = vf[2 * j + 1][0][x >> 1];
        f[j] = __builtin_amdgcn_perm(hi, lo, x & 1 ? 0x07060302u : 0x05040100u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = vf[4 * t + j][p][x];
    }
    return f;
  }
};

// Few queries, up to 16 (token, head) rows: the 4 waves of a workgroup take its 32-row tiles in turn, K and V from memory to
// registers without LDS, the page of the next tile's rows looked up by one lane each meanwhile.
// Bound by the bytes of K and V: 64 sequences of 16001 rows, D = 128 in bf16, 32 query and 8 KV heads, 667 us, 6.3 TB/s; of 1000
// to 16000 rows 348 us, 6.1 TB/s; one of 32768 rows 25 us, 5.4 TB/s, and 5 for the launch that joins the parts.  In fp32 one of
// 16000 rows 42 us, 3.1 TB/s; 32 of 1000 to 8000 rows 220 us, 5.5 TB/s.  Tried and no faster: K and V of a tile requested while
// the one before is worked on (31.3 for 32.2 us, fp32 121 for 107).
constexpr int kStreamRows = 16, kStreamTile = 32;

template <typename T, int D, bool kShare>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) void paged_stream_kernel(PagedAttendArgs a) {
  using W = PagedWave<T, D>;
  constexpr int TK = kStreamTile, kWaves = 4;
  __shared__ f32x4 so[2][W::NACC][64];
  __shared__ float sm[2][64], sl[2][64];
  __shared__ uint32_t scratch[8];
  const int lane = threadIdx.x & 63, i = lane & 15, c = lane >> 4, wave = wave_index();
  const T* K = static_cast<const T*>(a.k);
  const T* V = static_cast<const T*>(a.v);
  PagedShare s = paged_share<kStreamRows, TK, kShare>(a, scratch);
  const int g = s.g;
  paged_blocks<kStreamRows, TK, kShare>(a, s, [&](const PagedBlock<kStreamRows, TK>& blk, int u0, int u1, bool begins) {
    const int32_t* table = blk.table;
    const int r = blk.r0 + i;
    const bool valid = r < blk.R;
    const int t = valid ? divide(r, a.by_G) : 0;
    const int row = static_cast<int>(blk.q0 + t) * a.Hq + g * a.G + (r - t * a.G);     // where valid; below 2^29
    const int pos = valid ? blk.pos_of(a, r) : -1;
    auto row_of = [&](int u) -> uint32_t {                   // of row lane % 32 of the tile
      int base, from, to;
      blk.kt.tile(u, base, from, to);
      return page_row(a.pages, table, g, min(max(base + (lane & 31), from), to - 1));
    };
    const int u_end = min(u1, blk.kt.n);
    int u = u0 + wave;
    uint32_t rid = u < u_end ? row_of(u) : 0;
    // behind the look-up: loads return in the order of their requests
    W w;
    w.clear();
    w.load_q(static_cast<const T*>(a.q) + static_cast<int64_t>(valid ? row : 0) * D, valid, c);
    while (u < u_end) {
      u32x4 kf[2][W::NK];
      typename W::VPiece vf[8][W::NP];
      w.load_k(K, rid, i, c, kf);
      w.load_v(V, rid, i, c, vf);
      int base, from, to;
      blk.kt.tile(u, base, from, to);
      u += kWaves;
      if (u < u_end) rid = row_of(u);
      f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int kk = 0; kk < W::NK; ++kk)
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) mma_step<T>(sc[t2], kf[t2][kk], w.qf[kk]);
      w.template weigh<2>(sc, 0, base, from, to, pos, a, c);
      // The weights are rounded to the type of V, the precision the matrix cores take them in: each by 2^-8 of it at most in bf16,
      // to either side, so that a mean over many rows loses less.  Their sum is taken ahead of the rounding: the log-sum-exp, which
      // other calls join results and score rows by, is as exact as in fp32.
      if constexpr (W::kBf16) {
        const u32x4 pf = {pack_bf16x2(sc[0][0], sc[0][1]), pack_bf16x2(sc[0][2], sc[0][3]), pack_bf16x2(sc[1][0], sc[1][1]), pack_bf16x2(sc[1][2], sc[1][3])};
#pragma unroll
        for (int x = 0; x < W::NX; ++x) mma_step<T>(w.o[x], w.v_operand(vf, 0, x, 0), pf);
      } else {
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
          for (int p = 0; p < W::NP; ++p)
#pragma unroll
            for (int x = 0; x < W::NX; ++x) mma_step<T>(w.o[p * W::NX + x], w.v_operand(vf, p, x, t2), __builtin_bit_cast(u32x4, sc[t2]));
      }
    }
    // The four waves' shares, joined pairwise through LDS: (2, 3) into (0, 1), then 1 into 0.
    w.l = col4_sum(w.l);
#pragma unroll
    for (int half = 2; half >= 1; half >>= 1) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int x = 0; x < W::NACC; ++x) so[wave - half][x][lane] = w.o[x];
        sm[wave - half][lane] = w.m;
        sl[wave - half][lane] = w.l;
      }
      __syncthreads();
      if (wave < half) {
        const float m2 = sm[wave][lane], mn = fmaxf(w.m, m2), ref = mn == -INFINITY ? 0.f : mn;
        const float f = fast_exp2(w.m - ref), f2 = fast_exp2(m2 - ref);
        w.m = mn;
        w.l = w.l * f + sl[wave][lane] * f2;
#pragma unroll
        for (int x = 0; x < W::NACC; ++x) w.o[x] = w.o[x] * f + so[wave][x][lane] * f2;
      }
      __syncthreads();
    }
    const PagedTarget to = paged_target<kStreamRows, D, kShare>(a, s, blk, u0, u1, begins);
    if (wave == 0 && valid) w.write(to, a, row, i, c);
  });
}

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

// The stream of tiles into LDS, 16 bytes a lane and load: each of the 4 waves brings a quarter of a tile's rows, whose pages its
// lanes look up a tile ahead.  The 16-byte pieces of a row are permuted in LDS by XOR with the row.
template <typename T, int D>
struct PagedTiles {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int TK = kBf16 ? 64 : 32, kRows = kBf16 ? 128 : 64;
  static constexpr int kRowBytes = D * static_cast<int>(sizeof(T)), kChunks = kRowBytes / 16;
  static constexpr int kPerLoad = 64 / kChunks, kWaveRows = TK / 4, kLoads = kWaveRows / kPerLoad;      // rows of a load, of a wave
  static constexpr int kBytes = TK * kRowBytes;

  const PagedAttendArgs& a;
  const int32_t* table;
  int g, wave, lane;
  int entry, at_row;                                   // lane % kWaveRows: the page of one of the wave's rows of the tile looked up last

  __device__ __forceinline__ void look_up(const KeyTiles<TK>& kt, int u) {
    int base, from, to;
    kt.tile(u, base, from, to);
    const int p = min(max(base + kWaveRows * wave + lane % kWaveRows, from), to - 1);
    const int e = divide(p, a.pages.div);
    at_row = p - e * a.pages.page_size;
    entry = table[e];
  }
  // three at once: the rows of the first two, the third looked up
  __device__ __forceinline__ void look_up(const KeyTiles<TK>& kt, int u, int u2, int u3, uint32_t& first, uint32_t& second) {
    look_up(kt, u);
    const int e1 = entry, r1 = at_row;
    look_up(kt, u2);
    const int e2 = entry, r2 = at_row;
    look_up(kt, u3);
    const int e3 = entry, r3 = at_row;
    entry = e1; at_row = r1;
    first = row_number();
    entry = e2; at_row = r2;
    second = row_number();
    entry = e3; at_row = r3;
  }
  __device__ __forceinline__ uint32_t row_number() const {
    const int page = min(max(entry, 0), a.pages.n_pages - 1);
    return (static_cast<uint32_t>(page) * a.pages.Hkv + g) * a.pages.page_size + at_row;
  }
  // LDS serves 16 lanes of 16 bytes (32 of 8) at a time, from 64 banks, 256 bytes: of K those lanes have the same piece of 16 rows
  // in a row, of V (transposing reads) 64 bytes of 4 rows.  No conflicts so (45 % of the cycles that LDS was busy with K % 8 and
  // 2 (V % 4)).
  static __device__ __forceinline__ int swizzle_k(int r) { return kRowBytes == 128 ? (r >> 1) & 7 : r & 15; }
  static __device__ __forceinline__ int swizzle_v(int r) { return !kBf16 ? 0 : D == 128 ? 4 * (r & 3) : 2 * (r & 2); }
  // the wave's rows of K or V of a tile on their way to `dst`; swizzle(r), r the row among the wave's: XORed to the index of a
  // 16-byte piece
  template <typename S>
  __device__ __forceinline__ void issue(const void* src, uint32_t rid, char* dst, S&& swizzle) const {
    const int sub = lane / kChunks, piece = lane % kChunks;
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int r = n * kPerLoad + sub;                // of the wave's rows, whose number is a multiple of 8
      const int64_t off = static_cast<int64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(rid), r))) * kRowBytes;
      load_to_lds16(static_cast<const char*>(src) + off + (piece ^ swizzle(r)) * 16, dst + (kWaveRows * wave + n * kPerLoad) * kRowBytes);
    }
  }
  __device__ __forceinline__ void issue_k(uint32_t rid, char* dst) const {
    issue(a.k, rid, dst, [this](int r) { return swizzle_k(kWaveRows * wave + r); });
  }
  __device__ __forceinline__ void issue_v(uint32_t rid, char* dst) const {
    issue(a.v, rid, dst, [](int r) { return swizzle_v(r); });
  }
  __device__ __forceinline__ void landed() {
    stage_barrier();
    asm volatile("" : "+v"(entry));                    // looked at behind the wait of the barrier only
  }
};

__device__ __forceinline__ f32x16 mma32(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Many queries: the tiles of 64 rows go through LDS, where the 4 waves of a workgroup share them, 32 (token, head) rows of a
// group to a wave.  V of the next tile and K of the one behind it are on their way (straight into LDS, two buffers each) while
// one is worked on, and the next tile's logits are computed among its exponentials.
//
// S^T = K Q^T in products of 32 x 32 x 16: a lane has one query (l % 32) and of 32 rows the 16 rows 8 (r / 4) + 4 h + r % 4,
// h = l / 32.  Its weights are the B operand of O^T += V^T P^T as they are, since the order of the contraction is free: step s
// of 32 rows takes 16 s + 4 h + {0..3, 8..11} from lane half h.  V^T comes from LDS by transposing reads: 16 lanes name 4 rows
// x 4 pieces of 4 elements (lane i: row i / 4, piece i % 4) and get a column of 4 each; which elements of D make up the pieces
// is free too, and is taken so that a lane ends with 8 neighbouring elements of its query's output.
//
// Sums are taken against a reference that follows the maximum only when a tile exceeds it by 2^8 (any reference gives the
// same result while nothing overflows), so that the outputs are rarely rescaled.
//
// Bound by the chip's power: a prompt of 16384 tokens, D = 128, 32 query and 8 KV heads, runs at 2160 us, 1020 TFLOP/s, with the
// matrix cores busy half of the time at 1.75 GHz (a library's product of 8192 x 8192 matrices: 1314 TFLOP/s, 70 % at 1.67 GHz).
// What raises the share of the time lowers the clock: without the logits ahead 45 % at 1.86 GHz, 2230 us.
// (The shared forms keep 16 to 26 scalar registers in lanes of vector ones; no vector register is spilled.)
//
// Short prompts are bound by the chain of tiles of their last block, 1.35 us each where it has a compute unit to itself: 2048 tokens,
// 32 tiles, 56 us, 611 TFLOP/s; 4096 tokens 148 us, 930 TFLOP/s.
//
// Tried for 16384 tokens and no faster: schedules given to the compiler, 8 waves of 32 rows to a workgroup, 4 waves of 64 (half the
// reads of LDS, one wave on a SIMD and 36 % at 2.1 GHz: 2470 us; with D = 64 up to 10 % faster on prompts beyond 8000 tokens, 20 to 60 % slower on short ones).
template <int D, bool kShare>
__global__ __launch_bounds__(256, D == 64 && !kShare ? 3 : 2) void paged_tile_kernel(PagedAttendArgs a) {
  using P = PagedTiles<bf16_t, D>;
  constexpr int TK = P::TK, kRows = P::kRows, NS = D / 16, ND = D / 32;
  __shared__ __attribute__((aligned(16))) char s_k[2][P::kBytes], s_v[2][P::kBytes];
  const int lane = threadIdx.x & 63, wave = wave_index(), col = lane & 31, h = lane >> 5;
  PagedShare s = paged_share<kRows, TK, kShare>(a, reinterpret_cast<uint32_t*>(s_k[0]));
  const int g = s.g;
  // offsets of this lane's reads
  uint32_t k_off[NS], v_off[ND];
#pragma unroll
  for (int st = 0; st < NS; ++st) k_off[st] = col * P::kRowBytes + (((2 * st + h) ^ P::swizzle_k(col)) * 16);
  const int li = lane & 15, dh = (lane >> 4) & 1;
#pragma unroll
  for (int d = 0; d < ND; ++d)
    v_off[d] = (4 * h + (li >> 2)) * P::kRowBytes + (((4 * d + 2 * dh + (li & 1)) ^ P::swizzle_v(li >> 2)) * 16) + ((li & 3) >> 1) * 8;

  paged_blocks<kRows, TK, kShare>(a, s, [&](const PagedBlock<kRows, TK>& blk, int u0, int u1, bool begins) {
    // this wave's rows
    const int wr0 = blk.r0 + 32 * wave, r = wr0 + col;
    const bool valid = r < blk.R, any_rows = wr0 < blk.R;
    const int t = valid ? divide(r, a.by_G) : 0;
    const int row = static_cast<int>(blk.q0 + t) * a.Hq + g * a.G + (r - t * a.G);       // where valid; below 2^29
    const int pos = valid ? blk.pos_of(a, r) : -1;
    const int wave_min = blk.pos_of(a, wr0), wave_max = blk.pos_of(a, min(wr0 + 32, blk.R) - 1);
    P tiles{a, blk.table, g, wave, lane, 0, 0};
    const int u_end = min(u1, blk.kt.n);
    uint32_t first = 0, rid = 0;                         // this wave's rows of the tile that K was last requested of
    if (u0 < u_end) {
      tiles.look_up(blk.kt, u0, min(u0 + 1, u_end - 1), min(u0 + 2, u_end - 1), first, rid);
      tiles.issue_k(first, s_k[0]);
      tiles.issue_v(first, s_v[0]);
      if (u0 + 1 < u_end) tiles.issue_k(rid, s_k[1]);
    }
    // behind the look-up: loads return in the order of their requests
    u32x4 qf[NS];
#pragma unroll
    for (int st = 0; st < NS; ++st) qf[st] = valid ? ld16(static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(row) * D + st * 16 + h * 8) : zero16();
    f32x16 o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float ref = -INFINITY, l = 0.f;                      // reference (unscaled logits), this lane's share of the sum
    auto logits = [&](const char* __restrict kc, f32x16 (&sc)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[kb][e] = 0.f;
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const u32x4 kf = *reinterpret_cast<const u32x4*>(kc + k_off[st] + kb * 32 * P::kRowBytes);
          sc[kb] = mma32(kf, qf[st], sc[kb]);
        }
    };
    // tile u, whose logits are sc: the next tile's logits are computed (from kc) among the exponentials of this one's
    auto step = [&](int u, f32x16 (&sc)[2], f32x16 (&nx)[2], const char* __restrict kc, const char* __restrict vc, char* __restrict kn,
                    char* __restrict vn) __attribute__((always_inline)) {
      if (u + 1 < u_end) {
        tiles.issue_v(rid, vn);
        if (u + 2 < u_end) {
          rid = tiles.row_number();
          if (u + 3 < u_end) tiles.look_up(blk.kt, u + 3);
          tiles.issue_k(rid, kn);
        }
      }
      if (any_rows) {
        int base, from, to;
        blk.kt.tile(u, base, from, to);
        const bool full = base >= from && base + TK <= to && base + TK - 1 <= wave_min &&
                          (a.window == 0 || base > wave_max - a.window || base + TK <= a.sinks);
        if (!full) {
          // rows lo .. hi-1 of the cache, and where the range holds both, the first `sinks` rows
          const int lo = a.window ? max(from, pos - a.window + 1) : from, hi = min(to, pos + 1);
          const int first = base + 4 * h, sinks = a.window && base < a.sinks ? min(a.sinks, hi) : 0;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int j = first + (32 * kb + 8 * (e >> 2) + (e & 3));
              if (!((j >= lo && j < hi) || (j >= from && j < sinks))) sc[kb][e] = -INFINITY;
            }
        }
        float top = sc[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[kb][e]);
        float t0, t1;
        pair32(top, t0, t1);
        top = fmaxf(t0, t1);
        if (__any((top - ref) * a.sl2 > 8.f)) {          // -inf - -inf is no number and asks for nothing
          const float mn = fmaxf(ref, top), f = mn == ref ? 1.f : fast_exp2((ref - mn) * a.sl2);
          ref = mn;
          l *= f;
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] *= f;
        }
        const float shift = ref == -INFINITY ? 0.f : ref * a.sl2;
        // the matrix products of this wave ahead of the other's exponentials
        __builtin_amdgcn_s_setprio(1);
        logits(kc, nx);
        u32x4 pf[2][2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
          for (int e = 0; e < 16; ++e) { sc[kb][e] = fast_exp2(sc[kb][e] * a.sl2 - shift); l += sc[kb][e]; }
          // rounded to bf16, what the matrix cores take, after their sum, as in the streaming kernel
#pragma unroll
          for (int sh = 0; sh < 2; ++sh)
#pragma unroll
            for (int j = 0; j < 4; ++j) pf[kb][sh][j] = pack_bf16x2(sc[kb][8 * sh + 2 * j], sc[kb][8 * sh + 2 * j + 1]);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int sh = 0; sh < 2; ++sh)
#pragma unroll
            for (int d = 0; d < ND; ++d) {
              const char* vp = vc + v_off[d] + (32 * kb + 16 * sh) * P::kRowBytes;
              typedef __attribute__((address_space(3))) s16x4* LdsPtr;
              const s16x4 lo4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)vp);
              const s16x4 hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(vp + 8 * P::kRowBytes));
              const s16x8 vf = __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7);
              o[d] = mma32(__builtin_bit_cast(u32x4, vf), pf[kb][sh], o[d]);
            }
        __builtin_amdgcn_s_setprio(0);
      }
      tiles.landed();
    };
    if (u0 < u_end) {
      f32x16 sa[2], sb[2];
      tiles.landed();
      logits(s_k[0], sa);
      tiles.landed();                                    // the first step overwrites what was read here
      int u = u0;
      for (; u + 1 < u_end; u += 2) {
        step(u, sa, sb, s_k[1], s_v[0], s_k[0], s_v[1]);
        step(u + 1, sb, sa, s_k[0], s_v[1], s_k[1], s_v[0]);
      }
      if (u < u_end) step(u, sa, sb, s_k[1], s_v[0], s_k[0], s_v[1]);
    }
    const PagedTarget to = paged_target<kRows, D, kShare>(a, s, blk, u0, u1, begins);
    float lo, hi;
    pair32(l, lo, hi);
    l = lo + hi;
    const float m = ref * a.sl2;                           // log2 units
    if (!valid) return;
    if (to.final_rows) {
      const float inv = l > 0.f ? 1.f / l : 0.f;
      uint16_t* out = static_cast<uint16_t*>(a.out) + static_cast<int64_t>(row) * D;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 8) {
          u32x4 w;
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(o[d][e + 2 * j] * inv, o[d][e + 2 * j + 1] * inv);
          st16(out + 32 * d + 2 * e + 8 * h, w);
        }
      if (h == 0) a.lse[row] = l > 0.f ? (m + fast_log2(l)) * kLn2 : -INFINITY;
      return;
    }
    const int64_t at = to.by_row ? row : r - blk.r0;
    if (h == 0) to.ml[at] = float2{m, l};
    if (l == 0.f) return;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4*>(to.o + at * D + 32 * d + 16 * (e >> 3) + 8 * h + (e & 4)) = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
  });
}

// The same in fp32, tiles of 32 rows, products of 16 x 16 x 4: the layouts of the streaming kernel, with 16 rows to a wave and the
// operands read from LDS 16 rows of the cache at a time.  Logits, maximum, rescaling, weights and the product with V of 16 rows
// follow one another, and nothing but the other wave of a SIMD works meanwhile: D = 128, 32 query and 8 KV heads, a prompt of 4096
// tokens 1313 us, 105 TFLOP/s (a large fp32 matrix product: 153), 512 queries at 8192 rows 643 us, 104; a prompt of 1024 114 us, 75: a
// block's chain of tiles, 3 us each, shared out and joined.
template <int D, bool kShare>
__global__ __launch_bounds__(256, 2) void paged_tile32_kernel(PagedAttendArgs a) {
  using P = PagedTiles<float, D>;
  using W = PagedWave<float, D>;
  constexpr int TK = P::TK, kRows = P::kRows;
  __shared__ __attribute__((aligned(16))) char s_k[2][P::kBytes], s_v[2][P::kBytes];
  const int lane = threadIdx.x & 63, wave = wave_index(), i = lane & 15, c = lane >> 4;
  PagedShare s = paged_share<kRows, TK, kShare>(a, reinterpret_cast<uint32_t*>(s_k[0]));
  const int g = s.g;
  paged_blocks<kRows, TK, kShare>(a, s, [&](const PagedBlock<kRows, TK>& blk, int u0, int u1, bool begins) {
    const int wr0 = blk.r0 + 16 * wave, r = wr0 + i;
    const bool any_rows = wr0 < blk.R;
    const int wave_max = blk.pos_of(a, min(wr0 + 16, blk.R) - 1);
    const bool valid = r < blk.R;
    const int t0 = valid ? divide(r, a.by_G) : 0;
    const int row = static_cast<int>(blk.q0 + t0) * a.Hq + g * a.G + (r - t0 * a.G);     // where valid; below 2^29
    const int pos = valid ? blk.pos_of(a, r) : -1;
    P tiles{a, blk.table, g, wave, lane, 0, 0};
    const int u_end = min(u1, blk.kt.n);
    if (u0 < u_end) {
      uint32_t rid, none;
      tiles.look_up(blk.kt, u0, u0, min(u0 + 1, u_end - 1), rid, none);
      tiles.issue_k(rid, s_k[0]);
      tiles.issue_v(rid, s_v[0]);
    }
    W w;
    w.clear();
    w.load_q(static_cast<const float*>(a.q) + static_cast<int64_t>(valid ? row : 0) * D, valid, c);
    auto step = [&](int u, const char* __restrict kc, const char* __restrict vc, char* __restrict kn, char* __restrict vn) __attribute__((always_inline)) {
      if (u + 1 < u_end) {
        const uint32_t rid = tiles.row_number();
        if (u + 2 < u_end) tiles.look_up(blk.kt, u + 2);
        tiles.issue_k(rid, kn);
        tiles.issue_v(rid, vn);
      }
      int base, from, to;
      blk.kt.tile(u, base, from, to);
      if (any_rows && base <= wave_max) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < W::NK; ++kk)
            mma_step<float>(sc, *reinterpret_cast<const u32x4*>(kc + (16 * t + i) * P::kRowBytes + (((4 * kk + c) ^ P::swizzle_k(i)) * 16)), w.qf[kk]);
          w.template weigh<1>(&sc, t, base, from, to, pos, a, c);
#pragma unroll
          for (int p = 0; p < W::NP; ++p) {
            u32x4 vf[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) vf[y] = *reinterpret_cast<const u32x4*>(vc + (16 * t + 4 * c + y) * P::kRowBytes + p * 256 + i * 16);
#pragma unroll
            for (int x = 0; x < 4; ++x)
              mma_step<float>(w.o[p * 4 + x], u32x4{vf[0][x], vf[1][x], vf[2][x], vf[3][x]}, __builtin_bit_cast(u32x4, sc));
          }
        }
      }
      tiles.landed();
    };
    if (u0 < u_end) {
      tiles.landed();
      int u = u0;
      for (; u + 1 < u_end; u += 2) {
        step(u, s_k[0], s_v[0], s_k[1], s_v[1]);
        step(u + 1, s_k[1], s_v[1], s_k[0], s_v[0]);
      }
      if (u < u_end) step(u, s_k[0], s_v[0], s_k[1], s_v[1]);
    }
    const PagedTarget to = paged_target<kRows, D, kShare>(a, s, blk, u0, u1, begins);
    w.l = col4_sum(w.l);
    if (valid) w.write(to, a, row, r - blk.r0, c);
  });
}

// ---- joining the parts --------------------------------------------------------------------------------------------------

struct PagedJoinArgs {
  PagedAttendArgs a;
  int rows;                    // of a block
};

// The partial results of a (token, head) joined, by W waves: 1 where a workgroup joins four rows, more where rows are few and
// their parts many.  A part without any row of the cache has no output, only its (maximum, sum).
template <typename T, int D, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void paged_join_kernel(PagedJoinArgs j) {
  constexpr int N = D / 64, U = 4, kRowsHere = W == 1 ? 4 : 1;
  typedef float vec __attribute__((ext_vector_type(N)));
  const PagedAttendArgs& a = j.a;
  const int lane = threadIdx.x & 63, wave = wave_index(), part = wave % W;
  const int g = blockIdx.y, b = blockIdx.z, r = static_cast<int>(blockIdx.x) * kRowsHere + wave / W;
  int64_t q0;
  const int nq = query_range(a, b, q0), t = divide(r, a.by_G);
  if (t >= nq) return;
  const int64_t row = (q0 + t) * a.Hq + g * a.G + (r - t * a.G);
  // parts of the own block and of the prefix's: first workgroup, number, rows of the block
  int n[2] = {0, 0}, w0[2] = {0, 0}, which[2] = {0, 0}, br[2] = {0, 0};
#pragma unroll
  for (int sd = 0; sd < 2; ++sd) {
    if (sd == 1 && a.prefix_items == 0) continue;
    const int64_t at = sd == 0 ? r : q0 * a.G + r;
    n[sd] = 1;
    which[sd] = -1;                                        // a whole block
    if (a.share == 0) continue;
    const int block = static_cast<int>(at / j.rows);
    br[sd] = static_cast<int>(at - static_cast<int64_t>(block) * j.rows);
    const int4 cut = a.cut[sd == 0 ? a.prefix_items + b * a.blocks + block : block];
    w0[sd] = cut.x;
    n[sd] = cut.y - cut.x + 1;
    if (n[sd] > 1) which[sd] = cut.z;
  }
  if (a.prefix_items == 0 && which[0] < 0) return;         // already where it belongs
  const int slots = n[0] + n[1];
  float ref = -INFINITY, l = 0.f;
  vec o = 0.f;
  for (int base = 0; base < slots; base += 64) {
    const int at = base + lane;
    float2 ml{-INFINITY, 0.f};
    const float* po = nullptr;
    if (at < slots) {
      const int sd = at >= n[0], k = at - (sd ? n[0] : 0);
      if (which[sd] < 0) {
        const int64_t at2 = row + (sd ? a.total_q * a.Hq : 0);
        ml = a.whole_ml[at2];
        po = a.whole_o + at2 * D;
      } else {
        const int64_t slot = ((static_cast<int64_t>(g) * a.share + w0[sd] + k) * 2 + (k == 0 ? which[sd] : 0)) * j.rows + br[sd];
        ml = a.part_ml[slot];
        po = a.part_o + slot * D;
      }
    }
    float top = ml.x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float mn = fmaxf(ref, top), safe = mn == -INFINITY ? 0.f : mn;
    const float back = fast_exp2(ref - safe);
    const float f = ml.y > 0.f ? fast_exp2(ml.x - safe) : 0.f;
    ref = mn;
    l = l * back + wave_sum(ml.y * f);
    o *= back;
    const int here = min(64, slots - base);
    const uint64_t p64 = reinterpret_cast<uint64_t>(po);
    for (int k = part; k < here; k += W * U) {
      float w[U];
      vec v[U];
#pragma unroll
      for (int y = 0; y < U; ++y) {
        const int at2 = min(k + W * y, 63);
        w[y] = k + W * y < here ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), at2)) : 0.f;
        const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(p64), at2), hi = __builtin_amdgcn_readlane(static_cast<int>(p64 >> 32), at2);
        const float* src = reinterpret_cast<const float*>((static_cast<uint64_t>(hi) << 32) | lo);
        v[y] = 0.f;
        if (w[y] != 0.f) v[y] = *reinterpret_cast<const vec*>(src + lane * N);
      }
#pragma unroll
      for (int y = 0; y < U; ++y) o += v[y] * w[y];
    }
  }
  if constexpr (W > 1) {
    __shared__ vec so[W][64];
    so[part][lane] = o;
    __syncthreads();
    if (part != 0) return;
#pragma unroll
    for (int w = 1; w < W; ++w) o += so[w][lane];
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) store_elem(static_cast<T*>(a.out), row * D + lane * N + e, o[e] * inv);
  if (lane == 0) a.lse[row] = l > 0.f ? (ref + fast_log2(l)) * kLn2 : -INFINITY;
}

}  // namespace cd
